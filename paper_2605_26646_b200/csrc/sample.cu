// Next tokens from logits and given uniform numbers (unity_sample): temperature, top-k, top-p and min-p by a rule per role.
//
// Rows whose rule cuts nothing off take one pass over the logits (k_sample_stream, below); the others are searched (k_sample).
//
// k_sample: a cluster of blocks holds a row in shared memory: the logits cross HBM once and every further pass over them stays on chip.
// Thread order is index order (a thread owns `per` consecutive entries), so running masses are sums over threads.
//
// With x = (z - max z) / T and e = exp x, what is kept is a prefix of the entries in the order (logit falling, index rising),
// described by its last entry (logit, index).  min-p gives such a prefix at once, top-k by counting, top-p by mass.  Its end is
// enclosed by thresholds: a pass counts and weighs what is at or above two of them, and the next two come from the two before
// (for top-k first from the threads' largest entries, for top-p from mean and variance of x).  Once at most kList entries are
// left between two thresholds they are sorted; where a single value holds more, its entries go by index.
//
// A decision compares a sum of masses with a share of another.  Sums are taken of fp32 exponentials first, with a bound on
// their error (kSlackFast); where a comparison is closer than that, the row is done again with fp64 exponentials, so the outcome
// is that of 64-bit arithmetic either way.
#include "internal.h"
#include "ptx.cuh"

namespace unity {

namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxCluster = 16;
constexpr int kList = 1024;                  // entries sorted at most
constexpr int kTau = 2;                      // thresholds of a pass
constexpr float kLowest = -3.402823466e38f;
// fp32: e = ex2(z c - r), c = log2(e) / T, is off by 2^-22 of itself and, but for what all entries have in common, by the rounding of
// its argument and of c, 2^-24 |x| octaves each.  The mean of |x| under a distribution over 2^18 entries whose likeliest has p is at
// most h(p) + 18 (1 - p) + log2 p < 14: 1.16e-6.  8 or 16 values are added pairwise in fp32, the rest in fp64 or two parts: 2.4e-7.
// Both sides of a comparison carry that: 3.3e-6 of the whole mass.  fp64: 2^-48.
constexpr double kSlackFast = 3.3e-6, kSlackExact = 0.0;

struct Tally {                               // of the entries: mass of all, mass and number at or above each threshold
    double whole, m[kTau];
    float mean, square;                      // sums of e x and e x^2 (octaves)
    int c[kTau];
};
constexpr int kTallyWords = 2 + kTau + kTau / 2;
static_assert(sizeof(Tally) == 8 * kTallyWords && kTau % 2 == 0, "sent word by word");

struct Shared {
    uint64_t bar;                            // the row's arrival
    uint64_t mail[2];                        // the messages' arrival, of the even and of the odd exchanges
    unsigned long long box[2][kMaxCluster * kWarps];   // messages of every block, or of every warp
    Tally warp[kWarps];
    float warp_z[kWarps];
    int warp_n[kWarps];
    int scan[kWarps];
    double scan_m[kWarps];
    int found;
    double exp2_table[32];
    unsigned long long list[kList];          // (falling logit, rising index) as one rising number
};

// Messages between the blocks of a cluster: 8 bytes into another block's shared memory, counted by a barrier there.  An exchange is a
// set of messages with at least one from every block to every block, so no block is more than one exchange ahead of another: two
// barriers and two boxes, used in turn, do.
__device__ __forceinline__ void send(unsigned long long* slot, uint64_t* mail, int to, unsigned long long v) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];" ::"r"(ptx::mapa(ptx::smem_u32(slot), to)), "l"(v),
                 "r"(ptx::mapa(ptx::smem_u32(mail), to)) : "memory");
}
__device__ __forceinline__ bool mail_arrived(uint64_t* mail, unsigned parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(ptx::smem_u32(mail)), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ void wait_mail(uint64_t* mail, unsigned parity, int* status) {
    if (mail_arrived(mail, parity)) return;
    const long long t0 = clock64();
    while (!mail_arrived(mail, parity))
        if (clock64() - t0 > kWaitBudgetCycles) { atomicOr(status, kStatusTimeout); break; }
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}
// Inclusive sum over the lanes.
__device__ __forceinline__ double warp_scan(double v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double u = __shfl_up_sync(kFull, v, o);
        if (lane >= o) v += u;
    }
    return v;
}
// The larger one, NaN if one is NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
// Two neighbouring entries.
__device__ __forceinline__ float2 pair(const float* p) { return *reinterpret_cast<const float2*>(p); }
__device__ __forceinline__ float2 pair(const __nv_bfloat16* p) {
    const unsigned v = *reinterpret_cast<const unsigned*>(p);
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
__device__ __forceinline__ float one(const float* p) { return *p; }
__device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
// Order-preserving integers of floats, one for both zeros: neighbouring values have neighbouring integers.
__device__ __forceinline__ unsigned key_of(float z) {
    const unsigned b = __float_as_uint(z);
    return b >> 31 ? 0x80000000u - (b & 0x7fffffffu) : b + 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned k) {
    return __uint_as_float(k >= 0x80000000u ? k - 0x80000000u : 0x80000000u | (0x80000000u - k));
}

// exp((v - top) / T) in fp64 by a table (2^(j/32)) and the exponential series on a 64th of an octave: 2^k 2^(j/32) (1 + p), off
// by 2^-48; c64 = log2(e) / T.
__device__ __forceinline__ double slow_weight(float v, float top, double c64, double inv_t, const double* table) {
    const double d = static_cast<double>(v) - static_cast<double>(top), y = d * c64;    // (octaves; the largest logit's e is 1)
    if (!(y > -1020.0)) return v == -INFINITY ? 0.0 : exp(d * inv_t);
    constexpr double kShift = 0x1.8p52 / 32.0, kLn2 = 0.69314718055994531;              // the sum with kShift rounds to 32nds
    const double t = y + kShift, r = y - (t - kShift);
    const int n = __double2loint(t);                             // 32 k + j
    const double p = r * (kLn2 + r * (kLn2 * kLn2 / 2 + r * (kLn2 * kLn2 * kLn2 / 6 +
                          r * (kLn2 * kLn2 * kLn2 * kLn2 / 24 + r * (kLn2 * kLn2 * kLn2 * kLn2 * kLn2 / 120)))));
    const double b = table[n & 31];
    const double scaled = __hiloint2double(__double2hiint(b) + ((n >> 5) << 20), __double2loint(b));
    return fma(scaled, p, scaled);
}

__device__ __forceinline__ void put_row(const SampleArgs& a, int row, int token, double logp, double logp_kept, int n_kept) {
    a.token[row] = token;
    if (a.logp) a.logp[row] = static_cast<float>(logp);
    if (a.logp_kept) a.logp_kept[row] = static_cast<float>(logp_kept);
    if (a.n_kept) a.n_kept[row] = n_kept;
}
__device__ __forceinline__ void no_distribution(const SampleArgs& a, int row) { put_row(a, row, -1, NAN, NAN, 0); }
// The row's rule and number.  False: a row that is masked or has a bad role or number; its outputs are written here.
__device__ __forceinline__ bool row_begins(const SampleArgs& a, int row, int rank, SampleRule& rule, float& u) {
    const bool on = a.row_mask == nullptr || a.row_mask[row] != 0;
    const int role = a.row_role ? a.row_role[row] : 0;
    u = on ? a.u[row] : 0.f;
    if (on && role >= 0 && role < a.n_roles && u >= 0.f && u < 1.f) {
        rule = a.rules[role];
        return true;
    }
    if (rank == 0 && threadIdx.x == 0) {
        put_row(a, row, -1, 0.0, 0.0, 0);
        if (on) atomicOr(a.status, kStatusBadIndex);
    }
    return false;
}

// The kept entries end with (z, i).
struct Cut {
    float z;
    int i;
    __device__ __forceinline__ bool keeps(float v, int at) const { return v > z || (v == z && at <= i); }
};

template <typename T>
struct Row {
    Shared& s;
    T* z;                                    // the thread's entries
    int per, ctas, rank, first;              // entries of a thread (even); index of the thread's first entry in the row
    int* status;
    int turn;                                // exchanges so far
    int n_all, my_n;                         // entries above -inf, and the thread's own
    float top;                               // largest logit
    double inv_t, c64;                       // 1 / T, log2(e) / T
    float c, top_c;                          // log2(e) / T and that times the largest logit, in fp32
    double whole;                            // mass of all entries
    // what is known about the end of the kept entries: it lies in [lo, hi); the thread's own mass and numbers there
    float lo, hi;
    int n_lo, n_hi, my_lo, my_hi;
    double m_hi, my_m;
    float list_lo, list_hi;                  // the list holds the sorted entries of this interval
    bool cut_down;                           // entries were taken out of shared memory

    __device__ __forceinline__ int lane() const { return threadIdx.x & 31; }
    __device__ __forceinline__ int warp() const { return threadIdx.x >> 5; }

    // Weight of an entry.  -inf has none.
    __device__ __forceinline__ float octaves(float v) const { return fmaf(v, c, -top_c); }
    __device__ __forceinline__ float fast(float v) const { return ptx::ex2(octaves(v)); }
    __device__ __forceinline__ double slow(float v) const { return slow_weight(v, top, c64, inv_t, s.exp2_table); }
    template <bool EXACT>
    __device__ __forceinline__ double weight(float v) const { return EXACT ? slow(v) : static_cast<double>(fast(v)); }

    // One exchange: announce the bytes that will arrive here, send, wait.
    __device__ __forceinline__ uint64_t* mail() const { return &s.mail[turn & 1]; }
    __device__ __forceinline__ unsigned long long* box(int i) const { return &s.box[turn & 1][i]; }
    __device__ __forceinline__ void expect(int words) const {
        if (threadIdx.x == 0) ptx::mbar_arrive_expect_tx(mail(), 8 * words);
    }
    __device__ __forceinline__ void receive() { wait_mail(mail(), turn >> 1 & 1, status); ++turn; }
    // A word of every block to every block; returns the other side's place of it.  (Behind a barrier of the block.)
    __device__ __forceinline__ const unsigned long long* all_to_all(unsigned long long v) {
        const unsigned long long* got = box(0);
        expect(ctas);
        if (threadIdx.x < ctas) send(box(rank), mail(), threadIdx.x, v);
        receive();
        return got;
    }

    // Sums over the cluster, the same in every thread.
    __device__ __forceinline__ void add_lanes(Tally& v) const {
        v.whole = warp_sum(v.whole);
        v.mean = warp_sum(v.mean);
        v.square = warp_sum(v.square);
#pragma unroll
        for (int k = 0; k < kTau; ++k) {
            v.m[k] = warp_sum(v.m[k]);
            v.c[k] = __reduce_add_sync(kFull, v.c[k]);
        }
    }
    __device__ __forceinline__ Tally exchange(Tally v) {
        expect(ctas * kTallyWords);
        add_lanes(v);
        if (lane() == 0) s.warp[warp()] = v;
        __syncthreads();
        if (warp() == 0) {
            if (lane() < kWarps) v = s.warp[lane()]; else v = Tally{};
            add_lanes(v);
            if (lane() < ctas) {
                const unsigned long long* w = reinterpret_cast<const unsigned long long*>(&v);
#pragma unroll
                for (int i = 0; i < kTallyWords; ++i) send(box(rank * kTallyWords + i), mail(), lane(), w[i]);
            }
        }
        const Tally* got = reinterpret_cast<const Tally*>(box(0));
        receive();
        v = got[0];
        for (int r = 1; r < ctas; ++r) {
            v.whole += got[r].whole;
            v.mean += got[r].mean;
            v.square += got[r].square;
#pragma unroll
            for (int k = 0; k < kTau; ++k) { v.m[k] += got[r].m[k]; v.c[k] += got[r].c[k]; }
        }
        return v;
    }

    // One pass: mass of all entries, masses and numbers of those >= tau[k].  fp32: eight are added pairwise, their sums in two parts.
    template <bool EXACT, bool TAU, bool MOMENTS>
    __device__ __forceinline__ Tally weigh(const float (&tau)[kTau]) const {
        Tally v = {};
        float hi[kTau + 1] = {}, low[kTau + 1] = {};
        for (int j0 = 0; j0 < per; j0 += 8) {
            float x[8], e[8];
#pragma unroll
            for (int q = 0; q < 8; q += 2) {
                const float2 two = j0 + q < per ? pair(z + j0 + q) : make_float2(-INFINITY, -INFINITY);
                x[q] = two.x;
                x[q + 1] = two.y;
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                if (TAU)
#pragma unroll
                    for (int k = 0; k < kTau; ++k) v.c[k] += x[q] >= tau[k];
                if (EXACT) {
                    const double e64 = slow(x[q]);
                    v.whole += e64;
                    if (TAU)
#pragma unroll
                        for (int k = 0; k < kTau; ++k)
                            if (x[q] >= tau[k]) v.m[k] += e64;
                } else {
                    const float o = octaves(x[q]);
                    e[q] = ptx::ex2(o);
                    if (MOMENTS) {
                        const float eo = e[q] * fmaxf(o, -1e3f);
                        v.mean += eo;
                        v.square = fmaf(eo, fmaxf(o, -1e3f), v.square);
                    }
                }
            }
            if (!EXACT) {
#pragma unroll
                for (int k = 0; k <= (TAU ? kTau : 0); ++k) {
                    float f[8];
#pragma unroll
                    for (int q = 0; q < 8; ++q) f[q] = k == 0 || x[q] >= tau[k ? k - 1 : 0] ? e[q] : 0.f;
                    const float sum = ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
                    const float next = hi[k] + sum, part = next - hi[k];
                    low[k] += (hi[k] - (next - part)) + (sum - part);
                    hi[k] = next;
                }
            }
        }
        if (!EXACT) {
            v.whole = static_cast<double>(hi[0]) + static_cast<double>(low[0]);
#pragma unroll
            for (int k = 0; k < kTau; ++k) v.m[k] = static_cast<double>(hi[k + 1]) + static_cast<double>(low[k + 1]);
        }
        return v;
    }

    // A logit that about `want` entries or a few more reach: of every block its share of them is counted among its threads' largest
    // entries, and the least such logit is taken (blocks of less than half a share say nothing).  `mine`: the thread's largest.
    __device__ __forceinline__ float reached_by(int want, float mine, int valid, int V) {
        unsigned least = 0xffffffffu;
        if (2 * valid * ctas >= V) {
            const int n = static_cast<int>((static_cast<long long>(valid) * want + V - 1) / V);
            const unsigned key = mine > -INFINITY ? key_of(mine) : 0u;
            least = 0;
            for (int b = 31; b >= 14; --b) {                      // (the lower half of the digits says little)
                const unsigned next = least | 1u << b;
                if (__syncthreads_count(key >= next) >= n) least = next;
            }
        }
        __syncthreads();
        const unsigned long long* got = all_to_all(least);
        for (int r = 0; r < ctas; ++r) least = min(least, static_cast<unsigned>(got[r]));
        return least == 0u || least == 0xffffffffu ? -INFINITY : value_of(least);
    }

    // Exclusive prefix of `n` over the cluster's threads in index order.
    __device__ __forceinline__ int prefix(int n) {
        int v = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(kFull, v, o);
            if (lane() >= o) v += u;
        }
        if (lane() == 31) s.scan[warp()] = v;
        __syncthreads();
        const int w = lane() < kWarps ? s.scan[lane()] : 0;
        int before = v - n + __reduce_add_sync(kFull, lane() < warp() ? w : 0);
        const int block = __reduce_add_sync(kFull, w);
        const unsigned long long* got = all_to_all(block);
        for (int r = 0; r < rank; ++r) before += static_cast<int>(got[r]);
        return before;
    }

    // Encloses the end of the first k_want entries (BY_MASS false) or of the first whose mass reaches share of the whole, until at
    // most kList entries or one value are in [lo, hi).  `above`, `below`: first thresholds.  False: a comparison was too close for this
    // arithmetic.  (Every thread of the cluster gets the same result.)
    template <bool EXACT, bool BY_MASS>
    __device__ __forceinline__ bool enclose(int k_want, double share, float quantile, float above, float below, double* target, double* bound) {
        const double slack = EXACT ? kSlackExact : kSlackFast;
        const float octave = 0.69314718f / static_cast<float>(inv_t);
        float tau[kTau] = {above, below};
        double m_lo = 0.0;
        float centre = 0.f, width = 0.f;
        lo = kLowest;
        for (int round = 0;; ++round) {
            if (round > 0) {
                // between lo and hi: around the normal distribution's quantile, around the linear estimate, evenly; and evenly as
                // order-preserving integers where all that took long or the interval is far longer than the distribution
                const bool near = round < 10 && hi - lo < 256.f * octave;
                float at = 0.5f * (lo + hi), wide = (hi - lo) * (1.f / 6);
                if (BY_MASS && round == 1 && centre - width < hi && centre + width > lo) {
                    at = centre;
                    wide = width;
                } else if (BY_MASS && round < 5) {
                    at = hi - (hi - lo) * static_cast<float>((*target - m_hi) / (m_lo - m_hi));
                    wide = (hi - lo) * (round == 2 ? 0.1f : 0.04f);
                } else if (!BY_MASS && round < 5) {
                    at = hi - (hi - lo) * (static_cast<float>(k_want - n_hi) / static_cast<float>(n_lo - n_hi));
                    wide = (hi - lo) * 0.1f;
                }
                const unsigned a = key_of(lo), b = key_of(hi);
#pragma unroll
                for (int k = 0; k < kTau; ++k) {
                    const unsigned key = a + static_cast<unsigned>(static_cast<unsigned long long>(b - a) * (kTau - k) / (kTau + 1));
                    tau[k] = near || (BY_MASS && round == 1 && wide == width) ? (k == 0 ? at + wide : at - wide) : value_of(key);
                    if (!(tau[k] > lo && tau[k] < hi)) tau[k] = value_of(a + (b - a) / 2);
                }
            }
            const Tally mine = !EXACT && BY_MASS && round == 0 ? weigh<EXACT, true, true>(tau) : weigh<EXACT, true, false>(tau);
            const Tally v = exchange(mine);
            if (round == 0) {
                whole = v.whole;
                m_lo = v.whole;
                n_lo = n_all;
                my_lo = my_n;
                hi = nextafterf(top, INFINITY);
                n_hi = my_hi = 0;
                m_hi = my_m = 0.0;
                *target = share * v.whole;
                *bound = slack * v.whole;
                const float mean = v.mean / static_cast<float>(v.whole);
                const float sd = sqrtf(fmaxf(v.square / static_cast<float>(v.whole) - mean * mean, 0.f));
                centre = top + octave * (mean - sd * quantile);
                width = octave * (0.25f + 0.1f * sd);
            }
            bool moved = false;
#pragma unroll
            for (int k = 0; k < kTau; ++k) {
                if (!(tau[k] > lo && tau[k] < hi)) continue;
                const bool enough = BY_MASS ? v.m[k] >= *target + *bound : v.c[k] >= k_want;
                const bool little = BY_MASS ? v.m[k] < *target - *bound : v.c[k] < k_want;
                if (little) { hi = tau[k]; n_hi = v.c[k]; m_hi = v.m[k]; my_hi = mine.c[k]; my_m = mine.m[k]; moved = true; }
                else if (enough) { lo = tau[k]; n_lo = v.c[k]; m_lo = v.m[k]; my_lo = mine.c[k]; moved = true; }
            }
            if (n_lo - n_hi <= kList || key_of(hi) - key_of(lo) <= 1u) return true;
            if (!moved && round > 0) return false;
        }
    }

    // The entries in [lo, hi) in order: an entry's place is its rank behind the n_hi above.
    __device__ __forceinline__ void sort_list(int total) {
        if (list_lo == lo && list_hi == hi) return;
        list_lo = lo;
        list_hi = hi;
        int n = my_lo - my_hi, to = prefix(n);
        __syncthreads();                                          // (every warp has read its messages)
        expect(total + ctas);
        if (threadIdx.x < ctas) send(box(rank), mail(), threadIdx.x, 0);
        for (int j = 0; n > 0 && j < per; ++j) {
            const float x = one(z + j);
            if (!(x >= lo && x < hi)) continue;
            const unsigned long long item = static_cast<unsigned long long>(~key_of(x)) << 32 | static_cast<unsigned>(first + j);
            for (int r = 0; r < ctas; ++r) send(&s.list[to], mail(), r, item);
            ++to;
            --n;
        }
        int log_size = 6;
        while (1 << log_size < total) ++log_size;
        const int size = 1 << log_size;
        for (int i = total + threadIdx.x; i < size; i += kThreads) s.list[i] = ~0ull;
        receive();
        __syncthreads();
        // bitonic: a thread compares up to two pairs per step; up to 32 apart the pairs of a warp are the warp's own
        for (int k = 1; k <= log_size; ++k)
            for (int j = k - 1; j >= 0; --j) {
                for (int t = threadIdx.x; t < size / 2; t += kThreads) {
                    const int i = (t >> j << (j + 1)) | (t & ((1 << j) - 1));
                    const unsigned long long a = s.list[i], b = s.list[i + (1 << j)];
                    if ((a > b) == ((i >> k & 1) == 0)) { s.list[i] = b; s.list[i + (1 << j)] = a; }
                }
                if (j > 5 || (j > 0 ? j - 1 : k) > 5) __syncthreads(); else __syncwarp();
            }
        __syncthreads();
    }

    // Cuts the sorted entries: rank below k_want (behind the n_hi above) and, with BY_MASS, mass before them below the target.  With
    // k_want and a share the target is that share of the first k_want's mass.
    template <bool EXACT, bool BY_MASS>
    __device__ __forceinline__ bool cut_list(int total, int k_want, double share, double target, double bound, Cut* cut, int* n_kept) {
        constexpr int kEach = kList / kThreads;
        const int i0 = kEach * threadIdx.x;
        double e[kEach], sum = 0.0;
#pragma unroll
        for (int h = 0; h < kEach; ++h) {
            e[h] = BY_MASS && i0 + h < total && n_hi + i0 + h < k_want ? weight<EXACT>(value_of(~static_cast<unsigned>(s.list[i0 + h] >> 32))) : 0.0;
            sum += e[h];
        }
        double before = 0.0;
        if (BY_MASS) {
            const double run = warp_scan(sum, lane());
            if (lane() == 31) s.scan_m[warp()] = run;
            __syncthreads();
            const double w = lane() < kWarps ? s.scan_m[lane()] : 0.0;
            const double upto = warp_scan(w, lane());
            before = __shfl_sync(kFull, upto, warp() ? warp() - 1 : 0);
            before = (warp() ? before : 0.0) + (run - sum);
            if (share > 0.0) {
                const double all = __shfl_sync(kFull, upto, kWarps - 1);
                target = share * all;
                bound = (EXACT ? kSlackExact : kSlackFast) * all;
            }
        }
        int kept = 0;
        bool close = false;
#pragma unroll
        for (int h = 0; h < kEach; ++h) {
            if (i0 + h >= total || n_hi + i0 + h >= k_want) continue;
            const double m = m_hi + before;
            kept += !BY_MASS || m < target;
            close |= BY_MASS && !EXACT && fabs(m - target) <= bound && i0 + h + n_hi > 0;
            before += e[h];
        }
        const int warp_kept = __reduce_add_sync(kFull, kept);
        if (lane() == 0) s.scan[warp()] = warp_kept;
        if (__syncthreads_or(close)) return false;
        kept = __reduce_add_sync(kFull, lane() < kWarps ? s.scan[lane()] : 0);
        kept = kept > 0 ? kept : 1;                              // (rounding does not take the first one)
        const unsigned long long last = s.list[kept - 1];
        cut->z = value_of(~static_cast<unsigned>(last >> 32));
        cut->i = static_cast<int>(last & 0xffffffffu);
        *n_kept = n_hi + kept;
        return true;
    }

    // Cuts entries of one value, lo: so many of them by index.
    template <bool EXACT, bool BY_MASS>
    __device__ __forceinline__ bool cut_ties(int k_want, double target, double bound, Cut* cut, int* n_kept) {
        int want = k_want - n_hi;
        if (BY_MASS) {
            const double e = weight<EXACT>(lo), need = (target - m_hi) / e, up = ceil(need);
            if (!EXACT && !(fabs(need - rint(need)) * e > bound)) return false;
            want = !(up >= 1.0) ? 1 : up > n_lo - n_hi ? n_lo - n_hi : static_cast<int>(up);
        }
        want = min(want, n_lo - n_hi);
        const int n = my_lo - my_hi, before = prefix(n);
        if (threadIdx.x == 0) s.found = -1;
        __syncthreads();
        if (before < want && want <= before + n) {
            int left = want - before;
            for (int j = 0; j < per; ++j)
                if (one(z + j) == lo && --left == 0) { s.found = first + j; break; }
        }
        __syncthreads();
        const unsigned long long* got = all_to_all(static_cast<unsigned>(s.found + 1));
        int found = 0;
        for (int r = 0; r < ctas; ++r) found += static_cast<int>(got[r]);
        cut->z = lo;
        cut->i = found - 1;
        *n_kept = n_hi + want;
        return true;
    }

    // The first kept entry whose running mass is > u times the kept mass: those >= hi, and those in [lo, hi) that `cut` keeps.  The
    // warp that holds it writes the outputs.
    template <bool EXACT>
    __device__ __forceinline__ bool pick(const SampleArgs& a, int row, const Cut& cut, int n_kept, float u) {
        double mine = my_m;
        if (my_lo > my_hi)
            for (int j = 0; j < per; ++j) {
                const float x = one(z + j);
                if (x >= lo && x < hi && cut.keeps(x, first + j)) mine += weight<EXACT>(x);
            }
        const double run = warp_scan(mine, lane());               // inclusive over the warp's lanes
        const double sum = __shfl_sync(kFull, run, 31);
        expect(ctas * kWarps);
        if (lane() < ctas) send(box(rank * kWarps + warp()), mail(), lane(), static_cast<unsigned long long>(__double_as_longlong(sum)));
        const unsigned long long* region = box(0);
        receive();
        // Every warp looks for the warp whose range of running masses holds the target: the first that ends above it (u < 1, but
        // rounding may leave none: then the last with any mass).  A lane has four neighbouring warps.
        constexpr int kEach = kMaxCluster * kWarps / 32;
        double part[kEach], four = 0.0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int w = lane() * kEach + i;
            part[i] = w < ctas * kWarps ? __longlong_as_double(static_cast<long long>(region[w])) : 0.0;
            four += part[i];
        }
        const double upto = warp_scan(four, lane()), kept = __shfl_sync(kFull, upto, 31), prior = __shfl_up_sync(kFull, upto, 1);
        const double target = static_cast<double>(u) * kept, bound = EXACT ? kSlackExact : kSlackFast * kept;
        double from = lane() ? prior : 0.0, start = 0.0, last_start = 0.0;
        int hit = -1, last = -1;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const double to = from + part[i];
            if (part[i] > 0.0) {
                last = lane() * kEach + i;
                last_start = from;
                if (hit < 0 && to > target) { hit = last; start = from; }
            }
            from = to;
        }
        const unsigned hits = __ballot_sync(kFull, hit >= 0), lasts = __ballot_sync(kFull, last >= 0);
        const int owner = hits ? __ffs(hits) - 1 : 31 - __clz(lasts);
        const int home = __shfl_sync(kFull, hits ? hit : last, owner);
        start = __shfl_sync(kFull, hits ? start : last_start, owner);
        bool close = false;
        int token = -1;
        float tz = 0.f;
        if (home == rank * kWarps + warp()) {
            // in the warp the first lane whose running mass is above the target, of those with any
            const unsigned some = __ballot_sync(kFull, mine > 0.0), past = some & __ballot_sync(kFull, start + run > target);
            const int holder = past ? __ffs(past) - 1 : 31 - __clz(some);
            const double prev = __shfl_sync(kFull, run, holder ? holder - 1 : 0);
            double at0 = start + (holder ? prev : 0.0);
            close = fabs(at0 - target) <= bound;
            // its entries, 32 at a time
            const T* row_z = z + (holder - lane()) * per;
            const int base = first + (holder - lane()) * per;
            for (int j0 = 0; j0 < per; j0 += 32) {
                const int j = j0 + lane();
                float x = 0.f;
                double e = 0.0;
                if (j < per) {
                    x = one(row_z + j);
                    if (x >= hi || (x >= lo && cut.keeps(x, base + j))) e = weight<EXACT>(x);
                }
                const double at = at0 + warp_scan(e, lane());
                const unsigned any = __ballot_sync(kFull, e > 0.0), above = any & __ballot_sync(kFull, at > target);
                close |= __any_sync(kFull, e > 0.0 && fabs(at - target) <= bound);
                const int l = above ? __ffs(above) - 1 : any ? 31 - __clz(any) : -1;
                if (l >= 0) {
                    token = base + j0 + l;                        // (rounding may leave the last one below the target)
                    tz = __shfl_sync(kFull, x, l);
                }
                if (above) break;
                at0 = __shfl_sync(kFull, at, 31);
            }
        }
        if (!EXACT) {
            // (the block that holds the target decides for the cluster)
            const unsigned long long* got = all_to_all(__syncthreads_or(close) != 0);
            int sum_close = 0;
            for (int r = 0; r < ctas; ++r) sum_close += static_cast<int>(got[r]);
            if (sum_close > 0) return false;
        }
        if (token >= 0 && lane() == 0) {
            const double x = (static_cast<double>(tz) - static_cast<double>(top)) * inv_t;
            // fp32 weights have the largest logit's own in common, which rounding leaves next to 1
            const double common = EXACT ? 0.0 : 0.69314718055994531 * static_cast<double>(octaves(top));
            put_row(a, row, token, x + common - log(whole), x + common - log(kept), n_kept);
        }
        return true;
    }

    // Takes out of shared memory what `keep` refuses; what remains goes by the rest.
    template <typename F>
    __device__ __forceinline__ void reduce_to(int n, F keep) {
        my_n = 0;
        for (int j = 0; j < per; ++j) {
            const float x = one(z + j);
            if (keep(x, first + j)) my_n += x > -INFINITY;
            else z[j] = static_cast<T>(-INFINITY);
        }
        n_all = n;
        cut_down = true;
        list_lo = list_hi = 0.f;
        __syncwarp();                                             // (pick reads the entries of its warp's other lanes)
    }

    // floor: entries below it are not allowed (min-p).
    template <bool EXACT>
    __device__ __forceinline__ bool draw(const SampleArgs& a, int row, const SampleRule& rule, float floor, float my_top, int valid, float u) {
        const bool search = rule.top_k > 0 || rule.top_p < 1.0;
        Cut cut{kLowest, 0x7fffffff};                             // (every entry in [lo, hi))
        int n_kept = n_all;
        double all = -1.0;
        if (floor > -INFINITY) {
            // mass of all entries, and of those >= floor
            const float at[kTau] = {floor, INFINITY};
            const Tally mine = weigh<EXACT, true, false>(at), v = exchange(mine);
            whole = v.whole;
            lo = hi = floor;
            my_lo = my_hi = 0;
            my_m = mine.m[0];
            n_kept = v.c[0];
            if (!search) return pick<EXACT>(a, row, cut, n_kept, u);
            all = whole;
            reduce_to(n_kept, [&](float x, int) { return x >= floor; });
        }
        double target = 0.0, bound = 0.0;
        bool done = false;
        if (rule.top_k > 0) {
            const bool again = EXACT && list_lo < list_hi;        // the interval that the fp32 pass has found
            const float above = again ? list_hi : INFINITY, below = again ? list_lo : reached_by(rule.top_k, my_top, valid, a.V);
            if (!enclose<EXACT, false>(rule.top_k, 0.0, 0.f, above, below, &target, &bound)) return false;
            if (all < 0.0) all = whole;
            const int total = n_lo - n_hi;
            if (total <= kList) {
                // where all of the first k are in the list, top-p is decided there too
                sort_list(total);
                done = rule.top_p < 1.0 && n_hi == 0;
                if (done ? !cut_list<EXACT, true>(total, rule.top_k, rule.top_p, 0.0, 0.0, &cut, &n_kept)
                         : !cut_list<EXACT, false>(total, rule.top_k, 0.0, 0.0, 0.0, &cut, &n_kept)) return false;
            } else if (!cut_ties<EXACT, false>(rule.top_k, 0.0, 0.0, &cut, &n_kept)) return false;
            if (rule.top_p < 1.0 && !done)
                reduce_to(n_kept, [&](float x, int i) { return x >= hi || (x >= lo && cut.keeps(x, i)); });
        }
        if (rule.top_p < 1.0 && !done) {
            const bool again = EXACT && list_lo < list_hi;
            const float octave = 0.69314718f / static_cast<float>(inv_t);
            const float above = again ? list_hi : top - 2.f * octave, below = again ? list_lo : top - 10.f * octave;
            if (!enclose<EXACT, true>(0, rule.top_p, rule.quantile, above, below, &target, &bound)) return false;
            const int total = n_lo - n_hi;
            if (total <= kList) {
                sort_list(total);
                if (!cut_list<EXACT, true>(total, 0x7fffffff - kList, 0.0, target, bound, &cut, &n_kept)) return false;
            } else if (!cut_ties<EXACT, true>(0, target, bound, &cut, &n_kept)) return false;
        }
        if (all >= 0.0) whole = all;
        return pick<EXACT>(a, row, cut, n_kept, u);
    }
};

// The block's entries to shared memory: by one asynchronous copy where they begin at 16 bytes, -inf behind the row's end.
template <typename T>
__device__ __forceinline__ void fetch(Shared& s, T* z, const T* src, int n, int share, const SampleArgs& a) {
    const bool bulk = reinterpret_cast<uintptr_t>(src) % 16 == 0;
    const int whole = bulk ? n * static_cast<int>(sizeof(T)) / 16 * 16 / static_cast<int>(sizeof(T)) : 0;
    if (threadIdx.x == 0) {
        if (whole > 0) {
            ptx::mbar_arrive_expect_tx(&s.bar, whole * sizeof(T));
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(ptx::smem_u32(z)),
                         "l"(src), "r"(static_cast<uint32_t>(whole * sizeof(T))), "r"(ptx::smem_u32(&s.bar)) : "memory");
        }
    }
    if (!bulk) {
#pragma unroll 8
        for (int i = threadIdx.x; i < n; i += kThreads) z[i] = src[i];
    } else if (whole + static_cast<int>(threadIdx.x) < n) {
        z[whole + threadIdx.x] = src[whole + threadIdx.x];       // at most seven
    }
    for (int i = n + threadIdx.x; i < share; i += kThreads) z[i] = static_cast<T>(-INFINITY);
    __syncthreads();
    if (whole > 0 && !ptx::mbar_wait(&s.bar, 0, kWaitBudgetCycles)) atomicOr(a.status, kStatusTimeout);
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 4) k_sample(const __grid_constant__ SampleArgs a, int per, int ctas) {
    __shared__ Shared s;
    extern __shared__ __align__(16) unsigned char raw[];
    T* z = reinterpret_cast<T*>(raw);
    const int rank = ctas > 1 ? ptx::cluster_ctarank() : 0, row = blockIdx.x / ctas;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    SampleRule rule;
    float u;
    if (!row_begins(a, row, rank, rule, u) || !rule.search) return;           // (the same in every block of the cluster)
    if (threadIdx.x == 0) {
        ptx::mbar_init(&s.bar, 1);
        ptx::mbar_init(&s.mail[0], 1);
        ptx::mbar_init(&s.mail[1], 1);
        ptx::fence_barrier_init();
    }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // the block has begun and can take messages
    const int share = kThreads * per, begin = rank * share;
    const int n = a.V - begin < 0 ? 0 : a.V - begin < share ? a.V - begin : share;
    fetch(s, z, static_cast<const T*>(a.logits) + row * a.ld + begin, n, share, a);
    const int first = begin + static_cast<int>(threadIdx.x) * per;
    Row<T> r{s, z + threadIdx.x * per, per, ctas, rank, first, a.status, 0};

    // largest logit (NaN if one is NaN); entries above -inf
    float my_top = -INFINITY;
    int finite = 0;
    for (int j = 0; j < per; j += 2) {
        const float2 v = pair(r.z + j);
        my_top = max_nan(my_top, max_nan(v.x, v.y));
        finite += (v.x > -INFINITY) + (v.y > -INFINITY);
    }
    r.my_n = finite;
    float top = my_top;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(kFull, top, o));
    finite = __reduce_add_sync(kFull, finite);
    if (lane == 0) { s.warp_z[warp] = top; s.warp_n[warp] = finite; }
    __syncthreads();
    top = s.warp_z[0];
    finite = s.warp_n[0];
    for (int w = 1; w < kWarps; ++w) { top = max_nan(top, s.warp_z[w]); finite += s.warp_n[w]; }
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");     // before the first message
    const unsigned long long* got = r.all_to_all(static_cast<unsigned long long>(__float_as_uint(top)) << 32 | static_cast<unsigned>(finite));
    r.n_all = 0;
    for (int q = 0; q < ctas; ++q) {
        top = max_nan(top, __uint_as_float(static_cast<unsigned>(got[q] >> 32)));
        r.n_all += static_cast<int>(got[q] & 0xffffffffu);
    }
    if (!(top > -INFINITY && top < INFINITY)) {                   // NaN, +inf or nothing but -inf
        if (rank == 0 && threadIdx.x == 0) no_distribution(a, row);
        return;
    }
    r.top = top;
    r.inv_t = rule.inv_t;
    r.c64 = 1.4426950408889634 * rule.inv_t;
    r.c = static_cast<float>(r.c64);
    r.top_c = top * r.c;
    r.list_lo = r.list_hi = 0.f;
    r.cut_down = false;
    const int n_all = r.n_all, my_n = r.my_n;
    float floor = -INFINITY;
    if (rule.log_min_p > -INFINITY) {
        // the lowest logit with x >= log min_p
        const double want = static_cast<double>(top) + rule.log_min_p / rule.inv_t;
        floor = want > -3.4e38 ? static_cast<float>(want) : kLowest;
        auto passes = [&](float v) { return (static_cast<double>(v) - static_cast<double>(top)) * rule.inv_t >= rule.log_min_p; };
        for (int k = 0; k < 4 && floor > kLowest && passes(nextafterf(floor, -INFINITY)); ++k) floor = nextafterf(floor, -INFINITY);
        for (int k = 0; k < 4 && floor < top && !passes(floor); ++k) floor = nextafterf(floor, INFINITY);
    }
    // (fp32 weights have 2^(rounding of top_c) in common, which has to stay near 1)
    const bool fits = fabsf(r.top_c) <= 0x1p20f;
    if (fits && r.template draw<false>(a, row, rule, floor, my_top, n, u)) return;
    __syncthreads();
    if (threadIdx.x < 32) s.exp2_table[threadIdx.x] = exp2(threadIdx.x / 32.0);
    if (r.cut_down) {
        const T* src = static_cast<const T*>(a.logits) + row * a.ld + begin;
        for (int i = threadIdx.x; i < n; i += kThreads) z[i] = src[i];
        r.cut_down = false;
        r.list_lo = r.list_hi = 0.f;
        r.n_all = n_all;
        r.my_n = my_n;
    }
    __syncthreads();
    r.template draw<true>(a, row, rule, floor, my_top, n, u);
}

// ------------------------------------------------------------------------------------------------
// Rows whose rule leaves every entry (no top-k, top-p or min-p) and rows that take the largest logit: one pass over the logits in
// registers, no copy in shared memory, so that more rows are in flight.  Every warp of the cluster has a run of consecutive entries,
// in tiles of 512; a tile's masses refer to a power of two of its own next to its largest entry.  The warp whose running mass holds
// the target reads one of its tiles again.
// ------------------------------------------------------------------------------------------------
constexpr int kTileEntries = 512, kPerLane = kTileEntries / 32;
constexpr int kMaxTiles = 5;                 // of a warp
static_assert(kMaxTiles * kMaxCluster * kWarps * kTileEntries >= UNITY_MAX_SAMPLE_V, "enough for a row");

struct StreamShared {
    uint64_t mail[2];
    unsigned long long box[2][3 * kMaxCluster * kWarps];
    double tile_m[kWarps][kMaxTiles];        // mass of a tile, in units of 2^tile_r
    int tile_r[kWarps][kMaxTiles];
    double exp2_table[32];
};

template <typename T>
struct Tile {
    static constexpr int kVec = 16 / sizeof(T), kVecs = kPerLane / kVec;
    float v[kPerLane];
    static __device__ __forceinline__ int index(int base, int i) {               // of the lane's i-th entry
        return base + (i / kVec) * (32 * kVec) + (threadIdx.x & 31) * kVec + i % kVec;
    }
    __device__ __forceinline__ void load(const T* row, int base, int end, bool aligned) {
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
            const int at = index(base, k * kVec);
            if (aligned && at + kVec <= end) {
                const uint4 w = __ldg(reinterpret_cast<const uint4*>(row + at));
                const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (sizeof(T) == 4) v[k * kVec + q] = __uint_as_float(u[q]);
                    else {
                        v[k * kVec + 2 * q] = __uint_as_float(u[q] << 16);
                        v[k * kVec + (2 * q + 1) % kVec] = __uint_as_float(u[q] & 0xffff0000u);
                    }
                }
            } else {
#pragma unroll
                for (int q = 0; q < kVec; ++q) v[k * kVec + q] = at + q < end ? one(row + at + q) : -INFINITY;
            }
        }
    }
    __device__ __forceinline__ float largest() const {                            // NaN if one is NaN
        float m = v[0];
#pragma unroll
        for (int i = 1; i < kPerLane; ++i) m = max_nan(m, v[i]);
        return m;
    }
};
__device__ __forceinline__ double times_power(double m, int e) {                  // m 2^e, 0 far below
    return e < -1000 ? 0.0 : m * __hiloint2double((1023 + e) << 20, 0);
}

template <typename T>
struct Stream {
    StreamShared& s;
    const T* row;
    int ctas, rank, home, begin, end;        // the warp's number in the cluster and its entries [begin, end)
    bool aligned;
    int* status;
    int turn;
    float c;
    double c64, inv_t;
    float top;

    __device__ __forceinline__ int lane() const { return threadIdx.x & 31; }
    __device__ __forceinline__ int warp() const { return threadIdx.x >> 5; }
    __device__ __forceinline__ uint64_t* mail() const { return &s.mail[turn & 1]; }
    __device__ __forceinline__ unsigned long long* box(int i) const { return &s.box[turn & 1][i]; }
    __device__ __forceinline__ void expect(int words) const {
        if (threadIdx.x == 0) ptx::mbar_arrive_expect_tx(mail(), 8 * words);
    }
    __device__ __forceinline__ void receive() { wait_mail(mail(), turn >> 1 & 1, status); ++turn; }

    template <bool EXACT>
    __device__ __forceinline__ double weight(float v, int r) const {
        return EXACT ? slow_weight(v, top, c64, inv_t, s.exp2_table) : static_cast<double>(ptx::ex2(fmaf(v, c, -static_cast<float>(r))));
    }

    // Masses of the warp's tiles.
    template <bool EXACT>
    __device__ __forceinline__ void weigh_tile(const Tile<T>& t, int k, float most) {
        // (no finite entry: any unit will do)
        const int r = EXACT ? 0 : most > -INFINITY && most < INFINITY ? static_cast<int>(ceilf(fminf(fmaxf(most * c, -1e9f), 1e9f))) : 0;
        double m = 0.0;
        if (EXACT) {
#pragma unroll
            for (int i = 0; i < kPerLane; ++i) m += weight<true>(t.v[i], 0);
        } else {
            const float rf = static_cast<float>(r);
            float e[kPerLane];
#pragma unroll
            for (int i = 0; i < kPerLane; ++i) e[i] = ptx::ex2(fmaf(t.v[i], c, -rf));
#pragma unroll
            for (int o = kPerLane / 2; o > 0; o >>= 1)
#pragma unroll
                for (int i = 0; i < o; ++i) e[i] += e[i + o];
            m = static_cast<double>(e[0]);
        }
        m = warp_sum(m);
        if (lane() == 0) { s.tile_m[warp()][k] = m; s.tile_r[warp()][k] = r; }
    }

    // Sends the warp's mass, its unit, and two more numbers; finds the warp that holds the target and, there, the token.  `tz`: its
    // logit.  close: a comparison was too close for this arithmetic (known in that warp).
    struct Found { int token, n; float top, tz; int top_i, unit; double whole; bool close; };
    template <bool EXACT>
    __device__ __forceinline__ Found locate(int tiles, float my_top, int my_top_i, int my_n, float u) {
        __syncwarp();
        int r = -0x40000000;
        for (int k = 0; k < tiles; ++k)
            if (s.tile_m[warp()][k] > 0.0) r = max(r, s.tile_r[warp()][k]);
        double m = 0.0;
        for (int k = 0; k < tiles; ++k)
            if (s.tile_m[warp()][k] > 0.0) m += times_power(s.tile_m[warp()][k], s.tile_r[warp()][k] - r);
        const int warps = ctas * kWarps;
        expect(3 * warps);
        if (lane() < ctas) {
            send(box(3 * home), mail(), lane(), static_cast<unsigned long long>(__double_as_longlong(m)));
            send(box(3 * home + 1), mail(), lane(), static_cast<unsigned long long>(static_cast<unsigned>(r)) << 32 | static_cast<unsigned>(my_n));
            send(box(3 * home + 2), mail(), lane(), static_cast<unsigned long long>(__float_as_uint(my_top)) << 32 | static_cast<unsigned>(my_top_i));
        }
        const unsigned long long* got = box(0);
        receive();
        constexpr int kEach = kMaxCluster * kWarps / 32;
        Found f;
        f.token = -1;
        f.top = -INFINITY;
        f.top_i = 0x7fffffff;
        f.n = 0;
        f.unit = -0x40000000;
        f.close = false;
        f.tz = 0.f;
        double part[kEach], four = 0.0;
        int unit[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int w = lane() * kEach + i;
            part[i] = 0.0;
            unit[i] = -0x40000000;
            if (w < warps) {
                part[i] = __longlong_as_double(static_cast<long long>(got[3 * w]));
                unit[i] = static_cast<int>(got[3 * w + 1] >> 32);
                f.n += static_cast<int>(got[3 * w + 1] & 0xffffffffu);
                const float v = __uint_as_float(static_cast<unsigned>(got[3 * w + 2] >> 32));
                f.top_i = v > f.top ? static_cast<int>(got[3 * w + 2] & 0xffffffffu) : f.top_i;
                f.top = max_nan(f.top, v);
                f.unit = max(f.unit, unit[i]);
            }
        }
        f.unit = __reduce_max_sync(kFull, f.unit);
        f.n = __reduce_add_sync(kFull, f.n);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {                        // (the first of equal ones: lanes are in index order)
            const float v = __shfl_down_sync(kFull, f.top, o);
            const int i = __shfl_down_sync(kFull, f.top_i, o);
            if (lane() + o < 32) { f.top_i = v > f.top ? i : f.top_i; f.top = max_nan(f.top, v); }
        }
        f.top = __shfl_sync(kFull, f.top, 0);
        f.top_i = __shfl_sync(kFull, f.top_i, 0);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            part[i] = times_power(part[i], unit[i] - f.unit);
            four += part[i];
        }
        const double upto = warp_scan(four, lane()), prior = __shfl_up_sync(kFull, upto, 1);
        f.whole = __shfl_sync(kFull, upto, 31);
        const double target = static_cast<double>(u) * f.whole, bound = EXACT ? kSlackExact : kSlackFast * f.whole;
        double from = lane() ? prior : 0.0, start = 0.0, last_start = 0.0;
        int hit = -1, last = -1;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const double to = from + part[i];
            if (part[i] > 0.0) {
                last = lane() * kEach + i;
                last_start = from;
                if (hit < 0 && to > target) { hit = last; start = from; }
            }
            from = to;
        }
        const unsigned hits = __ballot_sync(kFull, hit >= 0), lasts = __ballot_sync(kFull, last >= 0);
        if (lasts == 0) return f;                                 // (a row without a distribution)
        const int owner = hits ? __ffs(hits) - 1 : 31 - __clz(lasts);
        const int holder = __shfl_sync(kFull, hits ? hit : last, owner);
        if (holder != home) return f;
        start = __shfl_sync(kFull, hits ? start : last_start, owner);
        // the tile: the first that ends above the target, or the last with any mass
        int tile = 0;
        double at0 = start;
        for (int k = 0; k < tiles; ++k) {
            const double mass = s.tile_m[warp()][k] > 0.0 ? times_power(s.tile_m[warp()][k], s.tile_r[warp()][k] - f.unit) : 0.0;
            if (!(mass > 0.0)) continue;
            tile = k;
            at0 = start;
            start += mass;
            if (start > target) break;
        }
        Tile<T> t;
        t.load(row, begin + tile * kTileEntries, end, aligned);
        f.close = fabs(at0 - target) <= bound;
        const int shift = s.tile_r[warp()][tile] - f.unit;
        // index order: vectors of the tile, lanes, entries of a lane
#pragma unroll
        for (int k = 0; k < Tile<T>::kVecs; ++k) {
            double e[Tile<T>::kVec], sum = 0.0;
#pragma unroll
            for (int q = 0; q < Tile<T>::kVec; ++q) {
                e[q] = times_power(weight<EXACT>(t.v[k * Tile<T>::kVec + q], s.tile_r[warp()][tile]), shift);
                sum += e[q];
            }
            double at = at0 + warp_scan(sum, lane()) - sum;       // before the lane's entries
            int mine = -1;
            float z = 0.f;
            bool over = false;
#pragma unroll
            for (int q = 0; q < Tile<T>::kVec; ++q) {
                at += e[q];
                if (e[q] > 0.0) {
                    f.close |= fabs(at - target) <= bound;
                    if (!over) {
                        mine = k * Tile<T>::kVec + q;
                        z = t.v[k * Tile<T>::kVec + q];
                        over = at > target;
                    }
                }
            }
            const unsigned any = __ballot_sync(kFull, mine >= 0), above = __ballot_sync(kFull, over);
            const int l = above ? __ffs(above) - 1 : any ? 31 - __clz(any) : -1;
            if (l >= 0) {
                const int i = __shfl_sync(kFull, mine, l);
                f.token = begin + tile * kTileEntries + (i / Tile<T>::kVec) * (32 * Tile<T>::kVec) + l * Tile<T>::kVec + i % Tile<T>::kVec;
                f.tz = __shfl_sync(kFull, z, l);
            }
            if (above) break;
            at0 = __shfl_sync(kFull, at, 31);
        }
        f.close = __any_sync(kFull, f.close);
        return f;
    }
};

template <typename T>
__global__ void __launch_bounds__(kThreads) k_sample_stream(const __grid_constant__ SampleArgs a, int run, int ctas) {
    __shared__ StreamShared s;
    const int rank = ctas > 1 ? ptx::cluster_ctarank() : 0, row = blockIdx.x / ctas;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    SampleRule rule;
    float u;
    if (!row_begins(a, row, rank, rule, u) || rule.search) return;            // (the same in every block of the cluster)
    if (threadIdx.x == 0) {
        ptx::mbar_init(&s.mail[0], 1);
        ptx::mbar_init(&s.mail[1], 1);
        ptx::fence_barrier_init();
    }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // the block has begun and can take messages
    const T* src = static_cast<const T*>(a.logits) + row * a.ld;
    const int home = rank * kWarps + warp, begin = home * run, end = min(a.V, begin + run);
    const int tiles = end > begin ? (end - begin + kTileEntries - 1) / kTileEntries : 0;
    Stream<T> r{s, src, ctas, rank, home, begin, end, reinterpret_cast<uintptr_t>(src) % 16 == 0, a.status, 0};
    r.inv_t = rule.inv_t;
    r.c64 = 1.4426950408889634 * rule.inv_t;
    r.c = static_cast<float>(r.c64);
    float top = -INFINITY;
    int top_i = 0x7fffffff, n = 0;
    for (int k = 0; k < tiles; ++k) {
        Tile<T> t;
        t.load(src, begin + k * kTileEntries, end, r.aligned);
        const float mine = t.largest();
        float most = mine;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) most = max_nan(most, __shfl_xor_sync(kFull, most, o));
        if (a.n_kept)
#pragma unroll
            for (int i = 0; i < kPerLane; ++i) n += t.v[i] > -INFINITY;
        if (rule.temperature == 0.f && most > top) {
            int at = 0x7fffffff;
#pragma unroll
            for (int i = kPerLane - 1; i >= 0; --i) at = t.v[i] == most ? Tile<T>::index(begin + k * kTileEntries, i) : at;
            top_i = __reduce_min_sync(kFull, at);
        }
        top = max_nan(top, most);
        r.template weigh_tile<false>(t, k, most);
    }
    n = __reduce_add_sync(kFull, n);
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");        // before the first message
    auto f = r.template locate<false>(tiles, top, top_i, n, u);
    if (!(f.top > -INFINITY && f.top < INFINITY)) {                  // NaN, +inf or nothing but -inf
        if (rank == 0 && threadIdx.x == 0) no_distribution(a, row);
        return;
    }
    // log of the whole mass: its unit, and what the rounding of c adds to every exponent alike
    const double shift = static_cast<double>(f.top) * (static_cast<double>(r.c) - r.c64);
    if (rule.temperature == 0.f) {
        if (rank == 0 && threadIdx.x == 0) {
            const double lse = (log2(f.whole) + f.unit - shift) * 0.69314718055994531;
            put_row(a, row, f.top_i, static_cast<double>(f.top) - lse, 0.0, 1);
        }
        return;
    }
    const bool fits = fabsf(f.top * r.c) <= 0x1p20f;                // (else a unit and c times a logit have no digits left to differ in)
    r.expect(ctas);
    const int close = __syncthreads_or(f.close || !fits);
    if (threadIdx.x < ctas) send(r.box(rank), r.mail(), threadIdx.x, close != 0);
    const unsigned long long* got = r.box(0);
    r.receive();
    int sum_close = 0;
    for (int q = 0; q < ctas; ++q) sum_close += static_cast<int>(got[q]);
    if (sum_close == 0) {
        if (f.token >= 0 && lane == 0) {
            const double logp = static_cast<double>(f.tz) * rule.inv_t - (log2(f.whole) + f.unit - shift) * 0.69314718055994531;
            put_row(a, row, f.token, logp, logp, f.n);
        }
        return;
    }
    __syncthreads();
    if (threadIdx.x < 32) s.exp2_table[threadIdx.x] = exp2(threadIdx.x / 32.0);
    __syncthreads();
    r.top = f.top;
    for (int k = 0; k < tiles; ++k) {
        Tile<T> t;
        t.load(src, begin + k * kTileEntries, end, r.aligned);
        r.template weigh_tile<true>(t, k, 0.f);
    }
    f = r.template locate<true>(tiles, top, top_i, n, u);
    if (f.token >= 0 && lane == 0) {
        const double logp = (static_cast<double>(f.tz) - static_cast<double>(f.top)) * rule.inv_t - log(f.whole);
        put_row(a, row, f.token, logp, logp, f.n);
    }
}

template <typename... P, typename... A>
cudaError_t launch_clusters(void (*kernel)(P...), int rows, int ctas, int bytes, cudaStream_t st, const A&... args) {
    cudaError_t e = bytes > 0 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) : cudaSuccess;
    if (e == cudaSuccess && ctas > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(rows) * ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, bool bf16, bool any_search, bool any_other, int sm_count, cudaStream_t st, int* n_launches) {
    if (any_other) {
        // a warp's run of entries: up to five tiles, and fewer while the rows leave SMs idle
        int ctas = 1, run = 0;
        for (;; ctas *= 2) {
            run = ((a.V + kWarps * ctas - 1) / (kWarps * ctas) + 7) / 8 * 8;
            if (ctas == kMaxCluster) break;
            if (run <= kMaxTiles * kTileEntries && (run <= kTileEntries || static_cast<long long>(a.n_rows) * ctas >= sm_count)) break;
        }
        const cudaError_t e = launch_clusters(bf16 ? k_sample_stream<__nv_bfloat16> : k_sample_stream<float>, a.n_rows, ctas, 0, st, a, run, ctas);
        if (e != cudaSuccess) return e;
        *n_launches += 1;
    }
    if (any_search) {
        // the fewest blocks per row (1 .. 16) whose share takes at most 40 KB, so that four blocks fit an SM
        const int width = bf16 ? 2 : 4;
        int ctas = 1, per = 0;
        for (;; ctas *= 2) {
            per = (a.V + kThreads * ctas - 1) / (kThreads * ctas);
            // entries are read in pairs, and the threads' first ones lie an odd number of pairs apart: at different banks
            per = ((per + 1) / 2 | 1) * 2;
            if (ctas == kMaxCluster || static_cast<long long>(per) * kThreads * width <= 40 * 1024) break;
        }
        const cudaError_t e = launch_clusters(bf16 ? k_sample<__nv_bfloat16> : k_sample<float>, a.n_rows, ctas, per * kThreads * width, st, a, per, ctas);
        if (e != cudaSuccess) return e;
        *n_launches += 1;
    }
    return cudaSuccess;
}

}  // namespace unity
