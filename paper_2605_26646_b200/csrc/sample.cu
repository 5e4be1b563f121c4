// Next tokens from logits and given uniform numbers (unity_sample): temperature, top-k, top-p and min-p by a rule per role.
//
// A cluster of blocks holds a row in shared memory: the logits cross HBM once and every further pass over them stays on chip.
// Thread order is index order (a thread owns `per` consecutive entries), so running masses are sums over threads.
//
// With x = (z - max z) / T and e = exp x, what is kept is a prefix of the entries in the order (logit falling, index rising),
// described by its last entry (logit, index).  min-p and top-k give such a prefix at once or by counting; top-p by mass.
// The prefix's end is searched by thresholds: a pass counts and weighs the entries at or above four of them, until at most
// kList entries are left between two, which are then ranked against one another, or only entries of one value, which go by index.
//
// A decision compares a sum of masses with a share of another.  Sums are taken in fp32 exponentials first, with a bound on
// their error (kSlack); where a comparison is closer than that, the row is done again with fp64 exponentials, so the outcome is
// that of 64-bit arithmetic either way.
#include "internal.h"
#include "ptx.cuh"

namespace unity {

namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kList = kThreads;              // entries ranked at most, one per thread
constexpr int kTau = 4;                      // thresholds of a pass
// fp32: e = ex2(x log2 e) is off by 2^-22 of itself, and by the roundings of x (twice 2^-24 |x|, whose mean under the
// distribution is at most 18 octaves at 2^18 entries: 1.5e-6); four values are added in fp32, the rest in fp64 (1.8e-7).  Both
// sides of a comparison carry that: 2^-18 of the whole mass.  fp64: exp is off by 2^-52 and by 2^-53 |x|.
constexpr double kSlackFast = 0x1p-18, kSlackExact = 0.0;

template <int N>
struct Sums {
    double m[N];
    int c[N];
};

struct Shared {
    Sums<kTau + 1> warp[kWarps];
    Sums<kTau + 1> cta[2][kMaxCluster];      // of every block of the cluster; two in turn: one cluster barrier per exchange
    double2 region[kMaxCluster * kWarps];    // (kept mass, whole mass) of every warp of the cluster
    int region_n[kMaxCluster * kWarps];
    float best_z[2][kMaxCluster];
    int best_i[2][kMaxCluster];
    float warp_z[kWarps];
    int warp_i[kWarps];
    int scan[kWarps];
    int count[2][kMaxCluster];
    int found;
    float list_z[kList];
    int list_i[kList];
    double list_e[kList];
    float last_z;
    int last_i;
};

__device__ __forceinline__ void remote_f64(void* local, int rank, double v) {
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(ptx::mapa(ptx::smem_u32(local), rank)), "d"(v) : "memory");
}
__device__ __forceinline__ void remote_u32(void* local, int rank, unsigned v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(ptx::mapa(ptx::smem_u32(local), rank)), "r"(v) : "memory");
}
__device__ __forceinline__ void cluster_meet() {
    __syncwarp();                            // (the barrier's instructions are for whole warps)
    ptx::cluster_sync_all();
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}
__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }
// Order-preserving integers of finite floats.
__device__ __forceinline__ unsigned key_of(float z) {
    const unsigned b = __float_as_uint(z);
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }

// The kept entries end with (z, i).
struct Cut {
    float z;
    int i;
    __device__ __forceinline__ bool keeps(float v, int at) const { return v > z || (v == z && at <= i); }
};

template <typename T>
struct Row {
    Shared& s;
    const T* z;                              // the block's entries
    int per, ctas, rank, first;              // entries of a thread; index of the thread's first entry in the row
    int turn, n_turn;
    float top;                               // largest logit
    double inv_t;
    float c_hi, c_lo;                        // log2(e) / T in two parts
    int V;

    __device__ __forceinline__ float at(int j) const { return as_float(z[threadIdx.x * per + j]) + 0.f; }   // (+ 0: -0 becomes 0)
    // Weight of an entry: fp32 or fp64 exponential.  -inf has none.
    template <bool EXACT>
    __device__ __forceinline__ double weight(float v) const {
        if (EXACT) return exp((static_cast<double>(v) - static_cast<double>(top)) * inv_t);
        return static_cast<double>(fast(v));
    }
    __device__ __forceinline__ float fast(float v) const {
        const float d = v - top;
        return ptx::ex2(fmaxf(fmaf(d, c_hi, d * c_lo), -200.f));
    }

    __device__ __forceinline__ Sums<kTau + 1> exchange(Sums<kTau + 1> v) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
        for (int k = 0; k <= kTau; ++k) {
            v.m[k] = warp_sum(v.m[k]);
            v.c[k] = __reduce_add_sync(kFull, v.c[k]);
        }
        if (lane == 0) s.warp[warp] = v;
        __syncthreads();
        if (threadIdx.x <= kTau) {
            const int k = threadIdx.x;
            double m = 0.0;
            int c = 0;
            for (int w = 0; w < kWarps; ++w) { m += s.warp[w].m[k]; c += s.warp[w].c[k]; }
            for (int r = 0; r < ctas; ++r) {
                remote_f64(&s.cta[turn][rank].m[k], r, m);
                remote_u32(&s.cta[turn][rank].c[k], r, c);
            }
        }
        cluster_meet();
        v = s.cta[turn][0];
        for (int r = 1; r < ctas; ++r)
#pragma unroll
            for (int k = 0; k <= kTau; ++k) { v.m[k] += s.cta[turn][r].m[k]; v.c[k] += s.cta[turn][r].c[k]; }
        turn ^= 1;
        return v;
    }

    // Number and mass of the entries that `cut` keeps and that are >= tau[k]; the last place: all that it keeps.
    template <bool EXACT>
    __device__ __forceinline__ Sums<kTau + 1> tally(const Cut& cut, const float (&tau)[kTau]) {
        Sums<kTau + 1> v = {};
        for (int j0 = 0; j0 < per; j0 += 4) {
            float part[kTau + 1] = {};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int j = j0 + q;
                if (j >= per) break;
                const float x = at(j);
                if (!cut.keeps(x, first + j)) continue;
                if (EXACT) {
                    const double e = weight<true>(x);
                    v.m[kTau] += e;
                    v.c[kTau] += 1;
#pragma unroll
                    for (int k = 0; k < kTau; ++k)
                        if (x >= tau[k]) { v.m[k] += e; v.c[k] += 1; }
                } else {
                    const float e = fast(x);
                    part[kTau] += e;
                    v.c[kTau] += 1;
#pragma unroll
                    for (int k = 0; k < kTau; ++k)
                        if (x >= tau[k]) { part[k] += e; v.c[k] += 1; }
                }
            }
            if (!EXACT)
#pragma unroll
                for (int k = 0; k <= kTau; ++k) v.m[k] += static_cast<double>(part[k]);
        }
        return exchange(v);
    }

    // Exclusive prefix of `n` over the cluster's threads in index order, and the total.
    __device__ __forceinline__ int prefix(int n, int* total) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        int v = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(kFull, v, o);
            if (lane >= o) v += u;
        }
        __syncthreads();
        if (lane == 31) s.scan[warp] = v;
        __syncthreads();
        int before = v - n, mine = 0;
        for (int w = 0; w < kWarps; ++w) { before += w < warp ? s.scan[w] : 0; mine += s.scan[w]; }
        if (threadIdx.x < ctas) remote_u32(&s.count[n_turn][rank], threadIdx.x, mine);
        cluster_meet();
        int all = 0;
        for (int r = 0; r < ctas; ++r) { before += r < rank ? s.count[n_turn][r] : 0; all += s.count[n_turn][r]; }
        n_turn ^= 1;
        *total = all;
        return before;
    }

    // Shortens `cut` to the first entries whose number reaches k (BY_MASS false) or whose mass reaches share * mass(cut).
    // False: a comparison was too close for this arithmetic.  (Every thread of the cluster gets the same result.)
    template <bool EXACT, bool BY_MASS>
    __device__ __forceinline__ bool shorten(Cut& cut, int k_want, double share) {
        const double slack = EXACT ? kSlackExact : kSlackFast;
        float lo = cut.z, hi = INFINITY;                         // the end lies in [lo, hi)
        int n_lo = 0, n_hi = 0;
        double m_hi = 0.0, target = 0.0, bound = 0.0;
        for (int round = 0;; ++round) {
            float tau[kTau];
            if (round == 0) {
                // octaves below the largest logit
                const float step = 0.69314718f / static_cast<float>(inv_t);
#pragma unroll
                for (int k = 0; k < kTau; ++k) tau[k] = top - step * (k == 0 ? 1.5f : k == 1 ? 5.f : k == 2 ? 9.f : 14.f);
            } else {
                // evenly between lo and hi, as values where they are close, else as order-preserving integers
                const unsigned a = key_of(lo), b = key_of(hi);
                const bool near = round < 6 && hi - lo < 64.f / static_cast<float>(inv_t);
#pragma unroll
                for (int k = 0; k < kTau; ++k) {
                    const unsigned key = a + static_cast<unsigned>(static_cast<unsigned long long>(b - a) * (kTau - k) / (kTau + 1));
                    tau[k] = near ? lo + (hi - lo) * (static_cast<float>(kTau - k) / (kTau + 1)) : value_of(key);
                    if (!(tau[k] > lo && tau[k] < hi)) tau[k] = value_of(a + 1);
                }
            }
            const Sums<kTau + 1> v = tally<EXACT>(cut, tau);
            if (round == 0) {
                n_lo = v.c[kTau];
                if (!BY_MASS && n_lo <= k_want) return true;      // nothing to cut off
                target = share * v.m[kTau];
                bound = slack * v.m[kTau];
                hi = nextafterf(top, INFINITY);
                if (!(lo > -INFINITY)) lo = -3.402823466e38f;
            }
            bool moved = false;
#pragma unroll
            for (int k = 0; k < kTau; ++k) {
                if (!(tau[k] > lo && tau[k] < hi)) continue;
                const bool enough = BY_MASS ? v.m[k] >= target + bound : v.c[k] >= k_want;
                const bool little = BY_MASS ? v.m[k] < target - bound || (EXACT && v.m[k] < target) : v.c[k] < k_want;
                if (little) { hi = tau[k]; n_hi = v.c[k]; m_hi = v.m[k]; moved = true; }
                else if (enough) { lo = tau[k]; n_lo = v.c[k]; moved = true; }
            }
            if (n_lo - n_hi <= kList || key_of(hi) - key_of(lo) <= 1u) break;
            if (!moved && round > 0) return false;
        }
        if (n_lo - n_hi <= kList) {
            // rank the entries in [lo, hi)
            int n = 0, total;
            for (int j = 0; j < per; ++j) {
                const float x = at(j);
                n += x >= lo && x < hi && cut.keeps(x, first + j);
            }
            int to = prefix(n, &total);
            for (int j = 0; j < per && n > 0; ++j) {
                const float x = at(j);
                if (!(x >= lo && x < hi && cut.keeps(x, first + j))) continue;
                const double e = BY_MASS ? weight<EXACT>(x) : 0.0;
                for (int r = 0; r < ctas; ++r) {
                    remote_u32(&s.list_z[to], r, __float_as_uint(x));
                    remote_u32(&s.list_i[to], r, first + j);
                    if (BY_MASS) remote_f64(&s.list_e[to], r, e);
                }
                ++to;
                --n;
            }
            cluster_meet();
            const int me = threadIdx.x;
            int before = 0;
            bool keep = false, close = false;
            if (me < total) {
                const float z0 = s.list_z[me];
                double mass = m_hi;
                for (int j = 0; j < total; ++j) {
                    const float z1 = s.list_z[j];
                    if (z1 > z0 || (z1 == z0 && j < me)) {        // (the list is in index order)
                        ++before;
                        if (BY_MASS) mass += s.list_e[j];
                    }
                }
                keep = BY_MASS ? mass < target : n_hi + before < k_want;
                close = BY_MASS && !EXACT && fabs(mass - target) <= bound;
            }
            const int kept = __syncthreads_count(keep);
            const bool too_close = __syncthreads_or(close);
            if (too_close) return false;
            if (keep && before == kept - 1) { s.last_z = s.list_z[me]; s.last_i = s.list_i[me]; }
            __syncthreads();
            cut.z = s.last_z;
            cut.i = s.last_i;
        } else {
            // entries of one value: so many of them by index
            int want = k_want - n_hi;
            if (BY_MASS) {
                const double e = weight<EXACT>(lo), need = (target - m_hi) / e, whole = ceil(need);
                if (!EXACT && !(fabs(need - rint(need)) * e > bound)) return false;
                want = !(whole >= 1.0) ? 1 : whole > n_lo - n_hi ? n_lo - n_hi : static_cast<int>(whole);
            }
            int n = 0, total;
            for (int j = 0; j < per; ++j) n += at(j) == lo && cut.keeps(lo, first + j);
            const int before = prefix(n, &total);
            if (before < want && want <= before + n) {
                int left = want - before, found = first;
                for (int j = 0; j < per; ++j)
                    if (at(j) == lo && cut.keeps(lo, first + j) && --left == 0) { found = first + j; break; }
                for (int r = 0; r < ctas; ++r) remote_u32(&s.found, r, found);
            }
            cluster_meet();
            cut.z = lo;
            cut.i = s.found;
        }
        return true;
    }

    // The first kept entry whose running mass is > u * mass(cut).  The thread that holds it writes the outputs.
    template <bool EXACT>
    __device__ __forceinline__ bool pick(const SampleArgs& a, int row, const Cut& cut, float u) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        double mine = 0.0, whole = 0.0;
        int n = 0;
        for (int j0 = 0; j0 < per; j0 += 4) {
            float kept4 = 0.f, all4 = 0.f;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int j = j0 + q;
                if (j >= per) break;
                const float x = at(j);
                const bool keep = cut.keeps(x, first + j);
                n += keep;
                if (EXACT) {
                    const double e = weight<true>(x);
                    whole += e;
                    mine += keep ? e : 0.0;
                } else {
                    const float e = fast(x);
                    all4 += e;
                    kept4 += keep ? e : 0.f;
                }
            }
            if (!EXACT) { whole += static_cast<double>(all4); mine += static_cast<double>(kept4); }
        }
        double run = mine;                                        // inclusive over the warp's lanes
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double v = __shfl_up_sync(kFull, run, o);
            if (lane >= o) run += v;
        }
        whole = warp_sum(whole);
        n = __reduce_add_sync(kFull, n);
        if (lane == 31)
            for (int r = 0; r < ctas; ++r) {
                remote_f64(&s.region[rank * kWarps + warp].x, r, run);
                remote_f64(&s.region[rank * kWarps + warp].y, r, whole);
                remote_u32(&s.region_n[rank * kWarps + warp], r, n);
            }
        cluster_meet();
        double before = 0.0, kept = 0.0;
        whole = 0.0;
        n = 0;
        for (int w = 0; w < ctas * kWarps; ++w) {
            if (w == rank * kWarps + warp) before = kept;
            kept += s.region[w].x;
            whole += s.region[w].y;
            n += s.region_n[w];
        }
        // The warp whose range of running masses holds the target; in it the first lane whose own does (rounding may leave that to a
        // lane without kept entries, or to none: then the next, or the last, with some).  u < 1, so the target is below kept.
        const double target = static_cast<double>(u) * kept, bound = EXACT ? kSlackExact : kSlackFast * kept;
        const double prev = __shfl_up_sync(kFull, run, 1);
        const double warp_end = before + __shfl_sync(kFull, run, 31);
        bool close = false;
        int token = -1;
        float tz = 0.f;
        if (before <= target && target < warp_end) {
            const unsigned some = __ballot_sync(kFull, mine > 0.0), past = some & __ballot_sync(kFull, before + run > target);
            if (lane == (past ? __ffs(past) - 1 : 31 - __clz(some))) {
                double c = before + (lane ? prev : 0.0);
                close = fabs(c - target) <= bound;
                for (int j = 0; j < per; ++j) {
                    const float x = at(j);
                    if (!cut.keeps(x, first + j)) continue;
                    const double e = weight<EXACT>(x);
                    if (!(e > 0.0)) continue;
                    token = first + j;
                    tz = x;
                    c += e;
                    close |= fabs(c - target) <= bound;
                    if (c > target) break;
                }
            }
        }
        if (!EXACT) {
            const bool any = __syncthreads_or(close);
            // (every block decides for the cluster: one more exchange)
            if (threadIdx.x < ctas) remote_u32(&s.count[n_turn][rank], threadIdx.x, any);
            cluster_meet();
            int sum = 0;
            for (int r = 0; r < ctas; ++r) sum += s.count[n_turn][r];
            n_turn ^= 1;
            if (sum > 0) return false;
        }
        if (token >= 0) {
            const double x = (static_cast<double>(tz) - static_cast<double>(top)) * inv_t;
            a.token[row] = token;
            if (a.logp) a.logp[row] = static_cast<float>(x - log(whole));
            if (a.logp_kept) a.logp_kept[row] = static_cast<float>(x - log(kept));
            if (a.n_kept) a.n_kept[row] = n;
        }
        return true;
    }

    template <bool EXACT>
    __device__ __forceinline__ bool draw(const SampleArgs& a, int row, const SampleRule& rule, Cut cut, float u) {
        if (rule.top_k > 0 && !shorten<EXACT, false>(cut, rule.top_k, 0.0)) return false;
        if (rule.top_p < 1.0 && !shorten<EXACT, true>(cut, 0, rule.top_p)) return false;
        return pick<EXACT>(a, row, cut, u);
    }
};

template <typename T>
__global__ void __launch_bounds__(kThreads) k_sample(const __grid_constant__ SampleArgs a, int per, int ctas) {
    __shared__ Shared s;
    extern __shared__ __align__(16) unsigned char raw[];
    T* z = reinterpret_cast<T*>(raw);
    const int rank = ctas > 1 ? ptx::cluster_ctarank() : 0, row = blockIdx.x / ctas;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool on = a.row_mask == nullptr || a.row_mask[row] != 0;
    const int role = a.row_role ? a.row_role[row] : 0;
    const float u = on ? a.u[row] : 0.f;
    if (!on || role < 0 || role >= a.n_roles || !(u >= 0.f && u < 1.f)) {     // (the same in every block of the cluster)
        if (rank == 0 && threadIdx.x == 0) {
            a.token[row] = -1;
            if (a.logp) a.logp[row] = 0.f;
            if (a.logp_kept) a.logp_kept[row] = 0.f;
            if (a.n_kept) a.n_kept[row] = 0;
            if (on) atomicOr(a.status, kStatusBadIndex);
        }
        return;
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // (the blocks of the cluster have begun: see below)
    const SampleRule rule = a.rules[role];
    const int share = kThreads * per, begin = rank * share;
    const T* src = static_cast<const T*>(a.logits) + row * a.ld + begin;
    const int n = a.V - begin < 0 ? 0 : a.V - begin < share ? a.V - begin : share;
    for (int i = threadIdx.x; i < share; i += kThreads) z[i] = i < n ? src[i] : static_cast<T>(-INFINITY);
    __syncthreads();
    Row<T> r{s, z, per, ctas, rank, begin + static_cast<int>(threadIdx.x) * per, 0, 0, 0.f, 0.0, 0.f, 0.f, a.V};

    // largest logit, the first of equal ones; a NaN makes it NaN
    float top = -INFINITY;
    int top_i = 0x7fffffff;
    bool bad = false;
    for (int j = 0; j < per; ++j) {
        const float x = r.at(j);
        bad |= !(x < INFINITY);
        if (x > top) { top = x; top_i = r.first + j; }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float v = __shfl_xor_sync(kFull, top, o);
        const int i = __shfl_xor_sync(kFull, top_i, o);
        if (v > top || (v == top && i < top_i)) { top = v; top_i = i; }
    }
    if (__any_sync(kFull, bad)) top = NAN;
    if (lane == 0) { s.warp_z[warp] = top; s.warp_i[warp] = top_i; }
    __syncthreads();
    top = s.warp_z[0];
    top_i = s.warp_i[0];
    bad = !(top == top);
    for (int w = 1; w < kWarps; ++w) {
        const float v = s.warp_z[w];
        bad |= !(v == v);
        if (v > top) { top = v; top_i = s.warp_i[w]; }
    }
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");     // before the first write to another block
    if (threadIdx.x < ctas) {
        remote_u32(&s.best_z[0][rank], threadIdx.x, __float_as_uint(bad ? NAN : top));
        remote_u32(&s.best_i[0][rank], threadIdx.x, top_i);
    }
    cluster_meet();
    top = -INFINITY;
    bad = false;
    for (int q = 0; q < ctas; ++q) {
        const float v = s.best_z[0][q];
        bad |= !(v == v);
        if (v > top) { top = v; top_i = s.best_i[0][q]; }
    }
    if (bad || !(top > -INFINITY)) {                              // NaN, +inf or nothing but -inf
        if (rank == 0 && threadIdx.x == 0) {
            a.token[row] = -1;
            if (a.logp) a.logp[row] = NAN;
            if (a.logp_kept) a.logp_kept[row] = NAN;
            if (a.n_kept) a.n_kept[row] = 0;
        }
        return;
    }
    r.top = top;
    r.inv_t = rule.inv_t;
    const double c = 1.4426950408889634 * rule.inv_t;
    r.c_hi = static_cast<float>(c);
    r.c_lo = static_cast<float>(c - static_cast<double>(r.c_hi));
    Cut cut{-INFINITY, -1};                                       // every entry above -inf
    SampleRule run = rule;
    if (rule.temperature == 0.f) {
        cut = Cut{top, top_i};                                    // (one entry is kept)
        run.top_k = 0;
        run.top_p = 1.0;
    } else if (rule.log_min_p > -INFINITY) {
        // the lowest logit with x >= log min_p
        double want = static_cast<double>(top) + rule.log_min_p / rule.inv_t;
        float least = want > -3.4e38 ? static_cast<float>(want) : -3.402823466e38f;
        auto passes = [&](float v) { return (static_cast<double>(v) - static_cast<double>(top)) * rule.inv_t >= rule.log_min_p; };
        for (int k = 0; k < 4 && least > -3.402823466e38f && passes(nextafterf(least, -INFINITY)); ++k) least = nextafterf(least, -INFINITY);
        for (int k = 0; k < 4 && least < top && !passes(least); ++k) least = nextafterf(least, INFINITY);
        cut = Cut{least + 0.f, 0x7fffffff};
    }
    if (!r.template draw<false>(a, row, run, cut, u)) r.template draw<true>(a, row, run, cut, u);
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, bool bf16, cudaStream_t st) {
    // the fewest blocks per row (1, 2, 4, 8) whose share takes at most 80 KB, so that two blocks fit an SM
    const int width = bf16 ? 2 : 4;
    int ctas = 1, per = 0;
    for (;; ctas *= 2) {
        per = (a.V + kThreads * ctas - 1) / (kThreads * ctas);
        // a thread's entries begin at different banks: an odd number of words apart
        per = bf16 ? ((per + 1) / 2 | 1) * 2 : per | 1;
        if (ctas == kMaxCluster || static_cast<long long>(per) * kThreads * width <= 80 * 1024) break;
    }
    const int bytes = per * kThreads * width;
    void (*kernel)(SampleArgs, int, int) = bf16 ? k_sample<__nv_bfloat16> : k_sample<float>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.n_rows) * ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, per, ctas);
}

}  // namespace unity
