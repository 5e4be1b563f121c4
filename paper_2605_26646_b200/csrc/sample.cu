// Next tokens from logits and given uniform numbers (unity_sample): temperature, top-k, top-p and min-p by a rule per role.
//
// Rows take one pass over the logits (k_sample_stream, below), at whose end a short list mostly decides where the rule cuts entries
// off; those that it cannot decide (flat ones by top-p, large top-k, masses too close) are searched (k_sample).
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
//
// What bounds it: latency for few rows (one of 152064 with top-k and top-p: 14 us, six exchanges of about 1.2 thousand clocks where the
// first list decides, among loads, a pass and a sort), issue slots for many (512 rows of 151936 fp32 with top-p of thirty thousand tokens:
// 900 us by the search alone, 1010 behind the pass, which does not decide such rows; the rows' bytes would take 48).  Four blocks per SM leave a
// thread 64 registers, so part of a row's state is in local memory (802 bytes of spill stores in the code for fp32, 878 for bf16); weighing
// is a function of its own so that its loop has none of it.
#include <algorithm>

#include "internal.h"
#include "ptx.cuh"

namespace unity {

namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxCluster = 16;
constexpr int kUnlisted = -2;                // a row's token between the two kernels: it is left to the search
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
    int c[kTau];
};
constexpr int kTallyWords = 1 + kTau + kTau / 2;
static_assert(sizeof(Tally) == 8 * kTallyWords && kTau % 2 == 0, "sent word by word");

struct Shared {
    uint64_t bar;                            // the row's arrival
    uint64_t mail[2];                        // the messages' arrival, of the even and of the odd exchanges
    unsigned long long box[2][kMaxCluster * kTallyWords];   // messages of every block
    Tally warp[kWarps];
    unsigned keys[kThreads];
    float warp_z[kWarps];
    int warp_n[kWarps];
    int scan[kWarps];
    double scan_m[kWarps];
    float2 moments[kWarps];
    int found;
    double exp2_table[32];
    uint16_t stage[kList];                   // the block's entries for the list, by their place in the block
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
// The largest of three, NaN if one is NaN; the least of three.
__device__ __forceinline__ float max_nan(float a, float b, float c) {
    float y;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ float min3(float a, float b, float c) {
    float y;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
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
__device__ __forceinline__ double slow_weight(float v, float top, double c64, const double* table) {
    const double d = static_cast<double>(v) - static_cast<double>(top), x = d * c64;    // (octaves; the largest logit's e is 1)
    // (no branch: neighbours are worked on together.  What lies between 2^-1075 and 2^-1020 is positive, all that is asked of it.)
    const double y = fmax(x, -1020.0);
    constexpr double kShift = 0x1.8p52 / 32.0, kLn2 = 0.69314718055994531;              // the sum with kShift rounds to 32nds
    const double t = y + kShift, r = y - (t - kShift);
    const int n = __double2loint(t);                             // 32 k + j
    const double p = r * (kLn2 + r * (kLn2 * kLn2 / 2 + r * (kLn2 * kLn2 * kLn2 / 6 +
                          r * (kLn2 * kLn2 * kLn2 * kLn2 / 24 + r * (kLn2 * kLn2 * kLn2 * kLn2 * kLn2 / 120)))));
    const double b = table[n & 31];
    const double scaled = __hiloint2double(__double2hiint(b) + ((n >> 5) << 20), __double2loint(b));
    return x < -1075.0 ? 0.0 : fma(scaled, p, scaled);
}

// m 2^e for e <= 0, 0 far below.
__device__ __forceinline__ double times_power(double m, int e) {                
    return e < -1000 ? 0.0 : m * __hiloint2double((1023 + e) << 20, 0);
}

// Lanes hold masses in index order: the first lane whose running mass (behind `before`) is above the target, or, where rounding leaves
// none, the last with any; its `start`: the mass before it.  -1: no mass at all.
__device__ __forceinline__ int owner(double mass, double before, double target, int lane, double* start) {
    const double upto = warp_scan(mass, lane), prior = __shfl_up_sync(kFull, upto, 1);
    const unsigned some = __ballot_sync(kFull, mass > 0.0), past = some & __ballot_sync(kFull, before + upto > target);
    if (some == 0) return -1;
    const int l = past ? __ffs(past) - 1 : 31 - __clz(some);
    *start = __shfl_sync(kFull, before + (lane ? prior : 0.0), l);
    return l;
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

// Sorts `total` numbers of a block's shared memory, room for kList of them: rising.
__device__ __forceinline__ void sort_items(unsigned long long* list, int total) {
    int log_size = 6;
    while (1 << log_size < total) ++log_size;
    const int size = 1 << log_size;
    for (int i = total + threadIdx.x; i < size; i += kThreads) list[i] = ~0ull;
    __syncthreads();
    if (total <= kThreads) {
        // each counts the smaller ones
        const unsigned long long mine = threadIdx.x < total ? list[threadIdx.x] : ~0ull;
        int below = 0;
        if (threadIdx.x < total)
#pragma unroll 8
            for (int i = 0; i < total; ++i) below += list[i] < mine;
        __syncthreads();
        if (threadIdx.x < total) list[below] = mine;
        __syncthreads();
        return;
    }
    // bitonic: a thread compares two pairs per step; up to 32 apart the pairs of a warp are the warp's own
    for (int k = 1; k <= log_size; ++k)
        for (int j = k - 1; j >= 0; --j) {
            for (int t = threadIdx.x; t < size / 2; t += kThreads) {
                const int i = (t >> j << (j + 1)) | (t & ((1 << j) - 1));
                const unsigned long long a = list[i], b = list[i + (1 << j)];
                if ((a > b) == ((i >> k & 1) == 0)) { list[i] = b; list[i + (1 << j)] = a; }
            }
            if (j > 5 || (j > 0 ? j - 1 : k) > 5) __syncthreads(); else __syncwarp();
        }
    __syncthreads();
}
// The lowest logit that min-p leaves, next to the largest one: (z - top) / T >= log min_p.
__device__ __forceinline__ float lowest_allowed(const SampleRule& rule, float top) {
    const double want = static_cast<double>(top) + rule.log_min_p / rule.inv_t;
    float floor = want > -3.4e38 ? static_cast<float>(want) : kLowest;
    auto passes = [&](float v) { return (static_cast<double>(v) - static_cast<double>(top)) * rule.inv_t >= rule.log_min_p; };
    for (int k = 0; k < 4 && floor > kLowest && passes(nextafterf(floor, -INFINITY)); ++k) floor = nextafterf(floor, -INFINITY);
    for (int k = 0; k < 4 && floor < top && !passes(floor); ++k) floor = nextafterf(floor, INFINITY);
    return floor;
}

// One pass over a thread's entries: mass of all, and with TAU masses and numbers of those >= tau[k].  fp32: two sums side by side (packed
// arithmetic), each of four entries added pairwise, those in two parts.  `moments`: sums of e x and e x^2 (octaves).
template <typename T, bool TAU, bool MOMENTS>
__device__ __forceinline__ Tally weigh_fast(const T* z, int per, float c, float top_c, float tau0, float tau1, float2* moments) {
    Tally v = {};
    float mean = 0.f, square = 0.f;
    const float tau[kTau] = {tau0, tau1};
    const uint64_t c2 = ptx::pack2(c, c), top2 = ptx::pack2(-top_c, -top_c), minus = ptx::pack2(-1.f, -1.f);
    uint64_t hi[kTau + 1] = {}, low[kTau + 1] = {};
    for (int j0 = 0; j0 < per; j0 += 8) {
        float x[8], e[8];
#pragma unroll
        for (int q = 0; q < 8; q += 2) {
            const float2 two = j0 + q < per ? pair(z + j0 + q) : make_float2(-INFINITY, -INFINITY);
            x[q] = two.x;
            x[q + 1] = two.y;
        }
        if constexpr (TAU) {
#pragma unroll
            for (int q = 0; q < 8; ++q)
#pragma unroll
                for (int k = 0; k < kTau; ++k) v.c[k] += x[q] >= tau[k];
        }
#pragma unroll
        for (int q = 0; q < 8; q += 2) {
            float a, b;
            ptx::unpack2(ptx::fma2(ptx::pack2(x[q], x[q + 1]), c2, top2), a, b);
            e[q] = ptx::ex2(a);
            e[q + 1] = ptx::ex2(b);
            if (MOMENTS) {
                a = fmaxf(a, -1e3f);
                b = fmaxf(b, -1e3f);
                mean += e[q] * a + e[q + 1] * b;
                square += e[q] * a * a + e[q + 1] * b * b;
            }
        }
#pragma unroll
        for (int k = 0; k <= (TAU ? kTau : 0); ++k) {
            uint64_t f[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float t = k ? tau[k - 1] : 0.f;
                f[q] = ptx::pack2(!k || x[2 * q] >= t ? e[2 * q] : 0.f, !k || x[2 * q + 1] >= t ? e[2 * q + 1] : 0.f);
            }
            const uint64_t sum = ptx::add2(ptx::add2(f[0], f[1]), ptx::add2(f[2], f[3])), next = ptx::add2(hi[k], sum);
            const uint64_t part = ptx::fma2(hi[k], minus, next);                           // next - hi
            const uint64_t lost = ptx::fma2(ptx::fma2(part, minus, next), minus, hi[k]);   // hi - (next - part)
            low[k] = ptx::add2(low[k], ptx::add2(lost, ptx::fma2(part, minus, sum)));
            hi[k] = next;
        }
    }
    if (MOMENTS) *moments = make_float2(mean, square);
#pragma unroll
    for (int k = 0; k <= (TAU ? kTau : 0); ++k) {
        float a, b, d, f;
        ptx::unpack2(hi[k], a, b);
        ptx::unpack2(low[k], d, f);
        (k ? v.m[k ? k - 1 : 0] : v.whole) = (static_cast<double>(a) + static_cast<double>(b)) + (static_cast<double>(d) + static_cast<double>(f));
    }
    return v;
}
// The same in fp64.
template <typename T, bool TAU>
__device__ __forceinline__ Tally weigh_slow(const T* z, int per, float top, double c64, const double* table, float tau0, float tau1) {
    Tally v = {};
    const float tau[kTau] = {tau0, tau1};
    for (int j0 = 0; j0 < per; j0 += 4) {
        float x[4];
        double w[4];
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
            const float2 two = j0 + q < per ? pair(z + j0 + q) : make_float2(-INFINITY, -INFINITY);
            x[q] = two.x;
            x[q + 1] = two.y;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = slow_weight(x[q], top, c64, table);
        v.whole += (w[0] + w[1]) + (w[2] + w[3]);
        if constexpr (TAU) {
#pragma unroll
            for (int k = 0; k < kTau; ++k)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    v.c[k] += x[q] >= tau[k];
                    v.m[k] += x[q] >= tau[k] ? w[q] : 0.0;
                }
        }
    }
    return v;
}
// As functions of their own, where much else is live: what a caller holds is put away once, not in the loop.
template <typename T>
__device__ __noinline__ Tally weigh_fast_apart(const T* z, int per, float c, float top_c, float tau0, float tau1) {
    return weigh_fast<T, true, false>(z, per, c, top_c, tau0, tau1, nullptr);
}
template <typename T, bool TAU>
__device__ __noinline__ Tally weigh_slow_apart(const T* z, int per, float top, double c64, const double* table, float tau0, float tau1) {
    return weigh_slow<T, TAU>(z, per, top, c64, table, tau0, tau1);
}

template <typename T>
struct Row {
    Shared& s;
    T* z;                                    // the thread's entries
    int per, ctas, rank, first;              // entries of a thread (even); index of the thread's first entry in the row
    int* status;
    int turn;                                // exchanges so far
    int n_all;                               // entries above -inf
    float top;                               // largest logit
    double inv_t, c64;                       // 1 / T, log2(e) / T
    float c, top_c;                          // log2(e) / T and that times the largest logit, in fp32
    double whole;                            // mass of all entries
    double my_all;                           // fp32: the thread's share of the mass of all entries of the row
    // what is known about the end of the kept entries: it lies in [lo, hi); the thread's own mass and numbers there
    float lo, hi;
    int n_lo, n_hi;
    double m_hi, my_m;
    unsigned long long marks[2];             // the thread's entries in [lo, hi)
    float list_lo, list_hi;                  // the list holds the sorted entries of this interval, list_n of them
    int list_n;
    bool cut_down;                           // entries were taken out of shared memory

    __device__ __forceinline__ int lane() const { return threadIdx.x & 31; }
    __device__ __forceinline__ int warp() const { return threadIdx.x >> 5; }

    // Weight of an entry.  -inf has none.
    __device__ __forceinline__ float octaves(float v) const { return fmaf(v, c, -top_c); }
    __device__ __forceinline__ float fast(float v) const { return ptx::ex2(octaves(v)); }
    __device__ __forceinline__ double slow(float v) const { return slow_weight(v, top, c64, s.exp2_table); }
    template <bool EXACT>
    __device__ __forceinline__ double weight(float v) const { return EXACT ? slow(v) : static_cast<double>(fast(v)); }

    // One exchange: announce the bytes that will arrive here, send, wait.
    __device__ __forceinline__ uint64_t* mail() const { return &s.mail[turn & 1]; }
    __device__ __forceinline__ unsigned long long* box(int i) const { return &s.box[turn & 1][i]; }
    __device__ __forceinline__ void expect(int words) const {
        if (threadIdx.x == 0) ptx::mbar_arrive_expect_tx(mail(), 8 * words);
    }
    // (One warp looks for the messages, the others wait at the block's barrier: looking takes issue slots.)
    __device__ __forceinline__ void receive() {
        if (warp() == 0) wait_mail(mail(), turn >> 1 & 1, status);
        __syncthreads();
        ++turn;
    }
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
        if (lane() < ctas) v = got[lane()]; else v = Tally{};
        add_lanes(v);
        return v;
    }

    template <bool EXACT, bool TAU, bool MOMENTS = false>
    __device__ __forceinline__ Tally weigh(const float (&tau)[kTau], float2* moments = nullptr) const {
        if constexpr (EXACT) return weigh_slow_apart<T, TAU>(z, per, top, c64, s.exp2_table, tau[0], tau[1]);
        else if constexpr (TAU) return weigh_fast_apart<T>(z, per, c, top_c, tau[0], tau[1]);
        else return weigh_fast<T, false, MOMENTS>(z, per, c, top_c, 0.f, 0.f, moments);
    }

    // A logit that about `want` entries or a few more reach: of every block its share of them is counted among its threads' largest
    // entries, and the least such logit is taken (blocks of less than half a share say nothing).  `mine`: the thread's largest.
    __device__ __forceinline__ float reached_by(int want, float mine, int valid, int V) {
        s.keys[threadIdx.x] = mine > -INFINITY ? key_of(mine) : 0u;
        __syncthreads();
        const unsigned long long* got = box(0);
        expect(ctas);
        if (warp() == 0) {
            unsigned least = 0xffffffffu;
            if (2 * valid * ctas >= V) {
                const int n = static_cast<int>((static_cast<long long>(valid) * want + V - 1) / V);
                unsigned key[kWarps];
#pragma unroll
                for (int i = 0; i < kWarps; ++i) key[i] = s.keys[32 * i + lane()];
                least = 0;
                for (int b = 31; b >= 14; --b) {                  // (the lower half of the digits says little)
                    const unsigned next = least | 1u << b;
                    int above = 0;
#pragma unroll
                    for (int i = 0; i < kWarps; ++i) above += key[i] >= next;
                    if (__reduce_add_sync(kFull, above) >= n) least = next;
                }
            }
            if (lane() < ctas) send(box(rank), mail(), lane(), least);
        }
        receive();
        const unsigned least = __reduce_min_sync(kFull, lane() < ctas ? static_cast<unsigned>(got[lane()]) : 0xffffffffu);
        return least == 0u || least == 0xffffffffu ? -INFINITY : value_of(least);
    }

    // Exclusive prefix of `n` over the cluster's threads in index order, and over the block's; the block's and the cluster's sum.
    struct Prefix { int cluster, block, block_n, n; };
    __device__ __forceinline__ Prefix prefix(int n) {
        int v = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(kFull, v, o);
            if (lane() >= o) v += u;
        }
        if (lane() == 31) s.scan[warp()] = v;
        __syncthreads();
        const int w = lane() < kWarps ? s.scan[lane()] : 0;
        Prefix p;
        p.block = v - n + __reduce_add_sync(kFull, lane() < warp() ? w : 0);
        p.block_n = __reduce_add_sync(kFull, w);
        const unsigned long long* got = all_to_all(p.block_n);
        const int theirs = lane() < ctas ? static_cast<int>(got[lane()]) : 0;
        p.cluster = p.block + __reduce_add_sync(kFull, lane() < rank ? theirs : 0);
        p.n = __reduce_add_sync(kFull, theirs);
        return p;
    }
    // Which of the thread's entries are in [lo, hi) (at most 128 of them).
    __device__ __forceinline__ int mark() {
        marks[0] = marks[1] = 0;
        for (int j0 = 0; j0 < per; j0 += 8) {
            unsigned m = 0;
#pragma unroll
            for (int q = 0; q < 8; q += 2) {
                const float2 two = j0 + q < per ? pair(z + j0 + q) : make_float2(-INFINITY, -INFINITY);
                m |= (two.x >= lo && two.x < hi ? 1u << q : 0u) | (two.y >= lo && two.y < hi ? 2u << q : 0u);
            }
            if (j0 < 64) marks[0] |= static_cast<unsigned long long>(m) << j0;
            else marks[1] |= static_cast<unsigned long long>(m) << (j0 - 64);
        }
        return __popcll(marks[0]) + __popcll(marks[1]);
    }
    template <typename F>
    __device__ __forceinline__ void each_marked(F f) const {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            for (unsigned long long m = marks[h]; m; m &= m - 1) f(64 * h + __ffsll(m) - 1);
    }

    // Encloses the end of the first k_want entries (BY_MASS false) or of the first whose mass reaches share of the whole, until at
    // most kList entries or one value are in [lo, hi).  `above`, `below`: first thresholds.  False: a comparison was too close for this
    // arithmetic.  (Every thread of the cluster gets the same result.)
    template <bool EXACT, bool BY_MASS>
    __device__ __forceinline__ bool enclose(int k_want, double share, float above, float below, double* target, double* bound) {
        const double slack = EXACT ? kSlackExact : kSlackFast;
        const float octave = 0.69314718f / static_cast<float>(inv_t);
        float tau[kTau] = {above, below};
        double m_lo = 0.0;
        lo = kLowest;
        for (int round = 0;; ++round) {
            if (round > 0) {
                // between lo and hi: around the linear estimate, evenly; and evenly as order-preserving integers where all that took long
                // or the interval is far longer than the distribution
                const bool near = round < 10 && hi - lo < 256.f * octave;
                float at = 0.5f * (lo + hi), wide = (hi - lo) * (1.f / 6);
                if (BY_MASS && round < 5) {
                    at = hi - (hi - lo) * static_cast<float>((*target - m_hi) / (m_lo - m_hi));
                    wide = (hi - lo) * (round == 1 ? 0.1f : 0.04f);
                } else if (!BY_MASS && round < 5) {
                    at = hi - (hi - lo) * (static_cast<float>(k_want - n_hi) / static_cast<float>(n_lo - n_hi));
                    wide = (hi - lo) * 0.1f;
                }
                const unsigned a = key_of(lo), b = key_of(hi);
#pragma unroll
                for (int k = 0; k < kTau; ++k) {
                    const unsigned key = a + static_cast<unsigned>(static_cast<unsigned long long>(b - a) * (kTau - k) / (kTau + 1));
                    tau[k] = near ? (k == 0 ? at + wide : at - wide) : value_of(key);
                    if (!(tau[k] > lo && tau[k] < hi)) tau[k] = value_of(a + (b - a) / 2);
                }
            }
            const Tally mine = weigh<EXACT, true>(tau);
            const Tally v = exchange(mine);
            if (round == 0) {
                whole = v.whole;
                m_lo = v.whole;
                n_lo = n_all;
                hi = nextafterf(top, INFINITY);
                n_hi = 0;
                m_hi = my_m = 0.0;
                *target = share * v.whole;
                *bound = slack * v.whole;
            }
            bool moved = false;
#pragma unroll
            for (int k = 0; k < kTau; ++k) {
                if (!(tau[k] > lo && tau[k] < hi)) continue;
                const bool enough = BY_MASS ? v.m[k] >= *target + *bound : v.c[k] >= k_want;
                const bool little = BY_MASS ? v.m[k] < *target - *bound : v.c[k] < k_want;
                if (little) { hi = tau[k]; n_hi = v.c[k]; m_hi = v.m[k]; my_m = mine.m[k]; moved = true; }
                else if (enough) { lo = tau[k]; n_lo = v.c[k]; m_lo = v.m[k]; moved = true; }
            }
            if (n_lo - n_hi <= kList || key_of(hi) - key_of(lo) <= 1u) return true;
            if (!moved && round > 0) return false;
        }
    }

    // The entries in [lo, hi) in order: an entry's place is its rank behind the n_hi above.  False: they are more than kList.
    __device__ __forceinline__ bool sort_list() {
        if (list_lo == lo && list_hi == hi) return true;
        const Prefix p = prefix(mark());
        if (p.n > kList) return false;
        list_n = p.n;
        list_lo = lo;
        list_hi = hi;
        const int total = p.n;
        int to = p.block;
        each_marked([&](int j) { s.stage[to++] = static_cast<uint16_t>(threadIdx.x * per + j); });
        __syncthreads();                                          // (and every warp has read its messages)
        expect(total + ctas);
        if (threadIdx.x < ctas) send(box(rank), mail(), threadIdx.x, 0);
        const int base = p.cluster - p.block, log_ctas = 31 - __clz(ctas);
        for (int i = threadIdx.x; i < p.block_n << log_ctas; i += kThreads) {
            const int k = i >> log_ctas, at = s.stage[k];
            const unsigned long long item = static_cast<unsigned long long>(~key_of(one(z - threadIdx.x * per + at))) << 32 |
                                            static_cast<unsigned>(first - threadIdx.x * per + at);
            send(&s.list[base + k], mail(), i & (ctas - 1), item);
        }
        receive();
        sort_items(s.list, total);
        return true;
    }

    // Cuts the sorted entries: rank below k_want (behind the n_hi above) and, with BY_MASS, mass before them below the target.  With
    // k_want and a share the target is that share of the first k_want's mass.
    enum Outcome { kDone, kClose, kShort };  // kShort: the list's mass does not reach the target
    template <bool EXACT, bool BY_MASS>
    __device__ __forceinline__ Outcome cut_list(int k_want, double share, double target, double bound, Cut* cut, int* n_kept) {
        constexpr int kEach = kList / kThreads;
        const int total = list_n;
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
            const double all = __shfl_sync(kFull, upto, kWarps - 1);
            if (share > 0.0) {
                target = share * all;
                bound = (EXACT ? kSlackExact : kSlackFast) * all;
            } else if (!(m_hi + all >= target + bound)) {
                return kShort;
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
        if (__syncthreads_or(close)) return kClose;
        kept = __reduce_add_sync(kFull, lane() < kWarps ? s.scan[lane()] : 0);
        kept = kept > 0 ? kept : 1;                              // (rounding does not take the first one)
        const unsigned long long last = s.list[kept - 1];
        cut->z = value_of(~static_cast<unsigned>(last >> 32));
        cut->i = static_cast<int>(last & 0xffffffffu);
        *n_kept = n_hi + kept;
        return kDone;
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
        const int n = mark(), before = prefix(n).cluster;
        if (threadIdx.x == 0) s.found = -1;
        __syncthreads();
        if (before < want && want <= before + n) {
            int left = want - before;
            each_marked([&](int j) { if (--left == 0) s.found = first + j; });
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
        each_marked([&](int j) {
            const float x = one(z + j);
            if (cut.keeps(x, first + j)) mine += weight<EXACT>(x);
        });
        const double run = warp_scan(mine, lane());               // inclusive over the warp's lanes
        if (lane() == 31) s.scan_m[warp()] = run;
        __syncthreads();
        const double of_warp = lane() < kWarps ? s.scan_m[lane()] : 0.0, of_block = warp_sum(of_warp);
        const unsigned long long* got = all_to_all(static_cast<unsigned long long>(__double_as_longlong(of_block)));
        const double block = lane() < ctas ? __longlong_as_double(static_cast<long long>(got[lane()])) : 0.0, kept = warp_sum(block);
        const double target = static_cast<double>(u) * kept, bound = EXACT ? kSlackExact : kSlackFast * kept;
        bool close = false;
        int token = -1;
        float tz = 0.f;
        double start = 0.0, logp = 0.0, logp_kept = 0.0;
        if (owner(block, 0.0, target, lane(), &start) == rank && owner(of_warp, start, target, lane(), &start) == warp()) {
            const int holder = owner(mine, start, target, lane(), &start);
            close = fabs(start - target) <= bound;
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
                const double at = start + warp_scan(e, lane());
                const unsigned any = __ballot_sync(kFull, e > 0.0), above = any & __ballot_sync(kFull, at > target);
                close |= __any_sync(kFull, e > 0.0 && fabs(at - target) <= bound);
                const int l = above ? __ffs(above) - 1 : any ? 31 - __clz(any) : -1;
                if (l >= 0) {
                    token = base + j0 + l;                        // (rounding may leave the last one below the target)
                    tz = __shfl_sync(kFull, x, l);
                }
                if (above) break;
                start = __shfl_sync(kFull, at, 31);
            }
            const double x = (static_cast<double>(tz) - static_cast<double>(top)) * inv_t;
            // fp32 weights have the largest logit's own in common, which rounding leaves next to 1
            const double common = EXACT ? 0.0 : 0.69314718055994531 * static_cast<double>(octaves(top));
            logp = x + common - log(whole);
            logp_kept = x + common - log(kept);
            if (!EXACT && tz == top) {
                // The likeliest entry may have nearly all of the mass: log p from what the others have, the sums without the thread's
                // share, and its other entries on their own (a sum of small ones next to a large one loses their digits)
                double others = 0.0, others_kept = 0.0;
                const T* all_z = static_cast<const T*>(a.logits) + row * a.ld;
                for (int j = lane(); j < per; j += 32) {
                    const int i = base + j;
                    if (i == token || i >= a.V) continue;
                    others += static_cast<double>(fast(one(all_z + i)));
                    const float v = one(row_z + j);
                    if (v >= hi || (v >= lo && cut.keeps(v, i))) others_kept += static_cast<double>(fast(v));
                }
                others = warp_sum(others) + (whole - __shfl_sync(kFull, my_all, holder));
                others_kept = warp_sum(others_kept) + (kept - __shfl_sync(kFull, mine, holder));
                const double own = static_cast<double>(fast(top));
                logp = 0.0 - log1p(fmax(others, 0.0) / own);
                logp_kept = 0.0 - log1p(fmax(others_kept, 0.0) / own);
            }
        }
        if (!EXACT) {
            // (the block that holds the target decides for the cluster)
            got = all_to_all(__syncthreads_or(close) != 0);
            if (__any_sync(kFull, lane() < ctas && got[lane() < ctas ? lane() : 0] != 0)) return false;
        }
        if (token >= 0 && lane() == 0) put_row(a, row, token, logp, logp_kept, n_kept);
        return true;
    }

    // Takes out of shared memory what `keep` refuses; what remains goes by the rest.
    template <typename F>
    __device__ __forceinline__ void reduce_to(int n, F keep) {
        for (int j = 0; j < per; ++j)
            if (!keep(one(z + j), first + j)) z[j] = static_cast<T>(-INFINITY);
        n_all = n;
        cut_down = true;
        list_lo = list_hi = 0.f;
        __syncwarp();                                             // (pick reads the entries of its warp's other lanes)
    }

    // floor: entries below it are not allowed (min-p).
    template <bool EXACT>
    __device__ __forceinline__ bool draw(const SampleArgs& a, int row, const SampleRule& rule, float floor, float my_top, int valid, float u, float centre, float width, bool spread) {
        const bool search = rule.top_k > 0 || rule.top_p < 1.0;
        Cut cut{kLowest, 0x7fffffff};                             // (every entry in [lo, hi))
        int n_kept = n_all;
        double all = -1.0;
        if (floor > -INFINITY) {
            // mass of all entries, and of those >= floor
            const float at[kTau] = {floor, INFINITY};
            const Tally mine = weigh<EXACT, true>(at), v = exchange(mine);
            whole = v.whole;
            my_all = mine.whole;
            lo = hi = floor;
            marks[0] = marks[1] = 0;
            my_m = mine.m[0];
            n_kept = v.c[0];
            if (!search) return pick<EXACT>(a, row, cut, n_kept, u);
            all = whole;
            whole = v.m[0];
            reduce_to(n_kept, [&](float x, int) { return x >= floor; });
        }
        if (EXACT && all < 0.0 && !(list_lo < list_hi && list_hi <= top)) {       // (else with the thresholds' pass)
            const float none[kTau] = {INFINITY, INFINITY};
            whole = exchange(weigh<true, false>(none)).whole;
        }
        const bool first_mass = all < 0.0;
        if (first_mass) all = whole;
        // What is kept is mostly among the first few hundred: those are sorted, and if they hold the end everything is decided there.
        // (Not where the distribution's entropy says that it is spread over many more.)
        const bool again = EXACT && list_lo < list_hi;            // the interval that the fp32 pass has found
        double target = rule.top_p * whole, bound = (EXACT ? kSlackExact : kSlackFast) * whole;
        float below = -INFINITY;
        bool done = false;
        if (rule.top_k <= kList / 4 * 3 && (rule.top_k > 0 || again || !spread)) {
            hi = nextafterf(top, INFINITY);
            n_hi = 0;
            m_hi = my_m = 0.0;
            if (again) {
                lo = list_lo;
                done = list_hi == hi;
            } else if (n_all <= kList) {
                lo = kLowest;
                done = true;
            } else {
                lo = below = reached_by(rule.top_k > 0 ? rule.top_k : kThreads / 2, my_top, valid, a.V);
                done = below > -INFINITY;
            }
            done = done && sort_list() && (rule.top_k == 0 || list_n >= min(rule.top_k, n_all));
            if (done) {
                const Outcome o = rule.top_k == 0 ? cut_list<EXACT, true>(0x7fffffff, 0.0, target, bound, &cut, &n_kept)
                                : rule.top_p < 1.0 ? cut_list<EXACT, true>(rule.top_k, rule.top_p, 0.0, 0.0, &cut, &n_kept)
                                                   : cut_list<EXACT, false>(rule.top_k, 0.0, 0.0, 0.0, &cut, &n_kept);
                if (o == kClose) return false;
                done = o == kDone;
            }
        }
        if (!done && rule.top_k > 0) {
            if (!enclose<EXACT, false>(rule.top_k, 0.0, again ? list_hi : INFINITY, again ? list_lo : below, &target, &bound)) return false;
            if (n_lo - n_hi <= kList) {
                sort_list();
                cut_list<EXACT, false>(rule.top_k, 0.0, 0.0, 0.0, &cut, &n_kept);
            } else {
                cut_ties<EXACT, false>(rule.top_k, 0.0, 0.0, &cut, &n_kept);
            }
            if (EXACT && first_mass) all = whole;
            if (rule.top_p < 1.0) reduce_to(n_kept, [&](float x, int i) { return x >= hi || (x >= lo && cut.keeps(x, i)); });
        }
        if (!done && rule.top_p < 1.0) {
            if (!enclose<EXACT, true>(0, rule.top_p, again ? list_hi : centre + width, again ? list_lo : centre - width, &target, &bound)) return false;
            if (EXACT && first_mass && rule.top_k == 0) all = whole;
            if (n_lo - n_hi <= kList) {
                sort_list();
                if (cut_list<EXACT, true>(0x7fffffff, 0.0, target, EXACT ? -1.0 : bound, &cut, &n_kept) != kDone) return false;
            } else if (!cut_ties<EXACT, true>(0, target, bound, &cut, &n_kept)) return false;
        }
        whole = all;
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
    if (threadIdx.x < 32 && whole > 0 && !ptx::mbar_wait(&s.bar, 0, kWaitBudgetCycles)) atomicOr(a.status, kStatusTimeout);
    __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 4) k_sample(const __grid_constant__ SampleArgs a, int per, int ctas, int listed) {
    __shared__ Shared s;
    extern __shared__ __align__(16) unsigned char raw[];
    T* z = reinterpret_cast<T*>(raw);
    const int rank = ctas > 1 ? ptx::cluster_ctarank() : 0, row = blockIdx.x / ctas;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    SampleRule rule;
    float u;
    if (listed) {
        ptx::grid_wait();                                                     // the pass is over
        if (a.token[row] != kUnlisted) return;                                // (no block writes before it hears from all of the cluster)
    }
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
    r.inv_t = rule.inv_t;
    r.c64 = 1.4426950408889634 * rule.inv_t;
    r.c = static_cast<float>(r.c64);
    // the mass, in units of a power of two next to the thread's largest entry
    int unit = my_top > -INFINITY && my_top < INFINITY ? static_cast<int>(ceilf(fminf(fmaxf(my_top * r.c, -1e9f), 1e9f))) : -1000000000;
    double mass = 0.0;
    float mean = 0.f, square = 0.f;
    if (rule.log_min_p == -INFINITY) {
        const float none[kTau] = {INFINITY, INFINITY};
        r.top_c = static_cast<float>(unit);
        float2 about = make_float2(0.f, 0.f);
        mass = rule.top_p < 1.0 ? r.template weigh<false, false, true>(none, &about).whole : r.template weigh<false, false>(none).whole;
        // (of the octaves themselves, no longer counted from the unit)
        const float f = static_cast<float>(unit), w = static_cast<float>(mass);
        mean = about.x + f * w;
        square = about.y + f * (2.f * about.x + f * w);
    }
    const double my_mass = mass;
    const int my_unit = unit;
    // Sums of masses in different units over the lanes of a warp.
    auto add_units = [&]() {
        const int most = __reduce_max_sync(kFull, unit), below = unit - most;
        const float scale = below < -100 ? 0.f : ptx::ex2(static_cast<float>(below));
        mass = warp_sum(times_power(mass, below));
        mean = warp_sum(scale * mean);
        square = warp_sum(scale * square);
        unit = most;
    };
    add_units();
    float top = my_top;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(kFull, top, o));
    finite = __reduce_add_sync(kFull, finite);
    if (lane == 0) { s.warp_z[warp] = top; s.warp_n[warp] = finite; s.scan_m[warp] = mass; s.scan[warp] = unit; s.moments[warp] = make_float2(mean, square); }
    __syncthreads();
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");     // before the first message
    r.expect(4 * ctas);
    if (warp == 0) {
        const bool on = lane < kWarps;
        top = on ? s.warp_z[lane] : -INFINITY;
        finite = on ? s.warp_n[lane] : 0;
        mass = on ? s.scan_m[lane] : 0.0;
        unit = on ? s.scan[lane] : -1000000000;
        mean = on ? s.moments[lane].x : 0.f;
        square = on ? s.moments[lane].y : 0.f;
        add_units();
#pragma unroll
        for (int o = kWarps / 2; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(kFull, top, o));
        top = __shfl_sync(kFull, top, 0);
        finite = __reduce_add_sync(kFull, finite);
        if (lane < ctas) {
            send(r.box(4 * rank), r.mail(), lane, static_cast<unsigned long long>(__float_as_uint(top)) << 32 | static_cast<unsigned>(finite));
            send(r.box(4 * rank + 1), r.mail(), lane, static_cast<unsigned long long>(__double_as_longlong(mass)));
            send(r.box(4 * rank + 2), r.mail(), lane, static_cast<unsigned>(unit));
            send(r.box(4 * rank + 3), r.mail(), lane, static_cast<unsigned long long>(__float_as_uint(mean)) << 32 | __float_as_uint(square));
        }
    }
    const unsigned long long* got = r.box(0);
    r.receive();
    {
        const bool on = lane < ctas;
        const unsigned long long* mine = got + 4 * (on ? lane : 0);
        top = on ? __uint_as_float(static_cast<unsigned>(mine[0] >> 32)) : -INFINITY;
        finite = on ? static_cast<int>(mine[0] & 0xffffffffu) : 0;
        mass = on ? __longlong_as_double(static_cast<long long>(mine[1])) : 0.0;
        unit = on ? static_cast<int>(mine[2]) : -1000000000;
        mean = on ? __uint_as_float(static_cast<unsigned>(mine[3] >> 32)) : 0.f;
        square = on ? __uint_as_float(static_cast<unsigned>(mine[3])) : 0.f;
        add_units();
#pragma unroll
        for (int o = kMaxCluster / 2; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(kFull, top, o));
        top = __shfl_sync(kFull, top, 0);
        r.n_all = __reduce_add_sync(kFull, finite);
    }
    if (!(top > -INFINITY && top < INFINITY)) {                   // NaN, +inf or nothing but -inf
        if (rank == 0 && threadIdx.x == 0) no_distribution(a, row);
        return;
    }
    r.top = top;
    r.top_c = top * r.c;
    const double to_top = exp2(static_cast<double>(unit) - static_cast<double>(r.top_c));
    r.whole = mass * to_top;
    r.my_all = times_power(my_mass, my_unit - unit) * to_top;
    // Where top-p ends in a normal distribution of the same mean and variance, and whether the entropy, log2 of the mass less the mean
    // in octaves below the largest, is that of more than some four hundred entries.  (Guesses.)
    mean /= static_cast<float>(mass);
    const float sd = sqrtf(fmaxf(square / static_cast<float>(mass) - mean * mean, 0.f));
    const float centre = (mean - sd * rule.quantile) / r.c, width = (0.25f + 0.1f * sd) / r.c;
    const bool spread = log2f(static_cast<float>(mass)) + static_cast<float>(unit) - mean > 8.6f;
    r.list_lo = r.list_hi = 0.f;
    r.cut_down = false;
    const int n_all = r.n_all;
    const float floor = rule.log_min_p > -INFINITY ? lowest_allowed(rule, top) : -INFINITY;
    // (fp32 weights have 2^(rounding of top_c) in common, which has to stay near 1)
    const bool fits = fabsf(r.top_c) <= 0x1p20f;
    if (fits && r.template draw<false>(a, row, rule, floor, my_top, n, u, centre, width, spread)) return;
    // the row in 64 bits
    __syncthreads();
    if (threadIdx.x < 32) s.exp2_table[threadIdx.x] = exp2(threadIdx.x / 32.0);
    if (r.cut_down) {
        const T* src = static_cast<const T*>(a.logits) + row * a.ld + begin;
        for (int i = threadIdx.x; i < n; i += kThreads) z[i] = src[i];
        r.cut_down = false;
        r.list_lo = r.list_hi = 0.f;
        r.n_all = n_all;
    }
    __syncthreads();
    r.template draw<true>(a, row, rule, floor, my_top, n, u, centre, width, spread);
}

// ------------------------------------------------------------------------------------------------
// Rows whose rule leaves every entry (no top-k, top-p or min-p) and rows that take the largest logit: one pass over the logits in
// registers, no copy in shared memory, so that more rows are in flight.  Every warp of the cluster has a run of consecutive entries,
// in tiles of 512; a lane's mass of a tile refers to a power of two next to the lane's largest entry there.  The warp whose running
// mass holds the target reads one of its tiles again.  512 rows of 151936: fp32 86 us (3.6 TB/s), bf16 61; each row ends with 6 to 8
// thousand clocks in which one warp of a block is at work, and rows whose decision is close (a third of flat ones) or whose largest entry
// lies so far from 0 that fp32 exponents have no digits left are read again.  Five blocks per SM leave a thread 48 registers (92 to 168
// bytes of spill stores in the code).
// ------------------------------------------------------------------------------------------------
constexpr int kTileEntries = 512, kPerLane = kTileEntries / 32;
constexpr int kMaxTiles = 20;                // of a warp
static_assert(kMaxTiles * kMaxCluster * kWarps * kTileEntries >= UNITY_MAX_SAMPLE_V, "enough for a row");

constexpr int kBins = 128, kListP = 128;      // (kListP: entries of a list for top-p, about)
struct ListState {                           // what a cluster's blocks know alike
    float top, floor;
    int unit, n_all, least, total, base;
    double whole, rest;
};
struct ListSpace {
    unsigned long long list[kList], stage[kList];
    uint16_t queue[kList];
};
struct StreamShared {
    uint64_t mail[2];
    unsigned long long box[2][4 * kMaxCluster];
    double warp_m[kWarps];                   // mass of a warp, in units of 2^warp_r
    int warp_r[kWarps], warp_n[kWarps], warp_i[kWarps];
    float warp_top[kWarps];
    float top;                               // what the first warp found out for the others
    int again;
    ListState known;
    int bins[kBins];                         // groups by their largest entry, in octaves below the block's largest
    int n_listed;
    double scan_a[kWarps], scan_b[kWarps];
    union {                                  // a lane's mass of a tile
        float2 lane_m[kMaxTiles][kThreads];  // x in units of 2^y
        double lane_x[kMaxTiles][kThreads];  // from fp64 weights, in units of 1
        ListSpace space;                     // (when the masses are no longer needed)
    };
    double exp2_table[32];
};

template <typename T>
struct Tile {
    static constexpr int kVec = 16 / sizeof(T), kVecs = kPerLane / kVec;
    uint4 raw[kVecs];
    static __device__ __forceinline__ int index(int base, int i) {               // of the lane's i-th entry
        return base + (i / kVec) * (32 * kVec) + (threadIdx.x & 31) * kVec + i % kVec;
    }
    __device__ __forceinline__ void load(const T* row, int base, int end, bool aligned) {
        if (aligned && base + kTileEntries <= end) {
            const uint4* p = reinterpret_cast<const uint4*>(row + base) + (threadIdx.x & 31);
#pragma unroll
            for (int k = 0; k < kVecs; ++k) raw[k] = __ldg(p + 32 * k);
            return;
        }
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
            const int at = index(base, k * kVec);
            if (aligned && at + kVec <= end) raw[k] = __ldg(reinterpret_cast<const uint4*>(row + at));
            else {
                unsigned w[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (sizeof(T) == 4) w[q] = at + q < end ? __float_as_uint(one(row + at + q)) : 0xff800000u;
                    else {
                        const unsigned lo = at + 2 * q < end ? __float_as_uint(one(row + at + 2 * q)) : 0xff800000u;
                        const unsigned hi = at + 2 * q + 1 < end ? __float_as_uint(one(row + at + 2 * q + 1)) : 0xff800000u;
                        w[q] = lo >> 16 | (hi & 0xffff0000u);
                    }
                }
                raw[k] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
    __device__ __forceinline__ void rotate() {                                    // the next vector becomes the first
#pragma unroll
        for (int k = 0; k + 1 < kVecs; ++k) raw[k] = raw[k + 1];
    }
    __device__ __forceinline__ float value(int i) const {
        const uint4& r = raw[i / kVec];
        const int q = i % kVec * sizeof(T) / 4;
        const unsigned w = q == 0 ? r.x : q == 1 ? r.y : q == 2 ? r.z : r.w;
        return __uint_as_float(sizeof(T) == 4 ? w : i % 2 ? w & 0xffff0000u : w << 16);
    }
};
template <typename T>
struct Stream {
    StreamShared& s;
    const T* row;
    int ctas, rank, run, V;                  // blocks of the cluster; entries of a warp
    bool aligned;
    int* status;
    int turn;
    float c;
    double c64, inv_t;
    float top;

    __device__ __forceinline__ int lane() const { return threadIdx.x & 31; }
    __device__ __forceinline__ int begin(int warp) const { return (rank * kWarps + warp) * run; }
    __device__ __forceinline__ int tiles(int warp) const {
        const int n = min(V, begin(warp) + run) - begin(warp);
        return n > 0 ? (n + kTileEntries - 1) / kTileEntries : 0;
    }
    __device__ __forceinline__ uint64_t* mail() const { return &s.mail[turn & 1]; }
    __device__ __forceinline__ unsigned long long* box(int i) const { return &s.box[turn & 1][i]; }
    __device__ __forceinline__ void expect(int words) const {
        if (threadIdx.x == 0) ptx::mbar_arrive_expect_tx(mail(), 8 * words);
    }
    __device__ __forceinline__ void receive() { wait_mail(mail(), turn >> 1 & 1, status); ++turn; }

    template <bool EXACT>
    __device__ __forceinline__ double weight(float v, int r) const {
        return EXACT ? slow_weight(v, top, c64, s.exp2_table) : static_cast<double>(ptx::ex2(fmaf(v, c, -static_cast<float>(r))));
    }
    // Unit of a lane's mass: the power of two at or above its largest entry (any, if it has none).
    __device__ __forceinline__ float unit_of(float most) const {
        return most > -INFINITY && most < INFINITY ? ceilf(fminf(fmaxf(most * c, -1e9f), 1e9f)) : -1e9f;
    }
    // The mass of tile k in lane `t` of the block, in units of 2^unit.
    template <bool EXACT>
    __device__ __forceinline__ double lane_mass(int k, int t, int unit) const {
        if (EXACT) return s.lane_x[k][t];
        const float2 m = s.lane_m[k][t];
        return times_power(static_cast<double>(m.x), static_cast<int>(m.y) - unit);
    }

    // One warp: the cluster's masses, and, in the block that holds the target, the token.  whole: in units of 2^unit; close: a
    // comparison was too close for this arithmetic (known in that block).
    struct Found { int token, n, top_i, unit; float top, tz; double whole; bool close; };
    template <bool EXACT>
    __device__ __forceinline__ Found locate(float u) {
        Found f;
        f.token = -1;
        f.tz = 0.f;
        f.close = false;
        // the block's sums
        const bool is_warp = lane() < kWarps;
        double m = is_warp ? s.warp_m[lane()] : 0.0;
        const int r = is_warp && m > 0.0 ? s.warp_r[lane()] : -0x40000000, block_r = __reduce_max_sync(kFull, r);
        float most = is_warp ? s.warp_top[lane()] : -INFINITY;
        int most_i = is_warp ? s.warp_i[lane()] : 0x7fffffff;
#pragma unroll
        for (int o = 1; o < kWarps; o <<= 1) {
            const float v = __shfl_down_sync(kFull, most, o);
            const int i = __shfl_down_sync(kFull, most_i, o);
            most_i = v > most ? i : most_i;                       // (lanes are in index order)
            most = max_nan(most, v);
        }
        most = __shfl_sync(kFull, most, 0);
        most_i = __shfl_sync(kFull, most_i, 0);
        const int n = __reduce_add_sync(kFull, is_warp ? s.warp_n[lane()] : 0);
        m = times_power(m, r - block_r);
        const double block_m = warp_sum(m);
        expect(3 * ctas);
        if (lane() < ctas) {
            send(box(3 * rank), mail(), lane(), static_cast<unsigned long long>(__double_as_longlong(block_m)));
            send(box(3 * rank + 1), mail(), lane(), static_cast<unsigned long long>(static_cast<unsigned>(block_r)) << 32 | static_cast<unsigned>(n));
            send(box(3 * rank + 2), mail(), lane(), static_cast<unsigned long long>(__float_as_uint(most)) << 32 | static_cast<unsigned>(most_i));
        }
        const unsigned long long* got = box(0);
        receive();
        double mass = 0.0;
        int unit = -0x40000000, count = 0;
        most = -INFINITY;
        most_i = 0x7fffffff;
        if (lane() < ctas) {
            mass = __longlong_as_double(static_cast<long long>(got[3 * lane()]));
            unit = static_cast<int>(got[3 * lane() + 1] >> 32);
            count = static_cast<int>(got[3 * lane() + 1] & 0xffffffffu);
            most = __uint_as_float(static_cast<unsigned>(got[3 * lane() + 2] >> 32));
            most_i = static_cast<int>(got[3 * lane() + 2] & 0xffffffffu);
        }
        f.unit = __reduce_max_sync(kFull, unit);
        f.n = __reduce_add_sync(kFull, count);
#pragma unroll
        for (int o = 1; o < kMaxCluster; o <<= 1) {
            const float v = __shfl_down_sync(kFull, most, o);
            const int i = __shfl_down_sync(kFull, most_i, o);
            most_i = v > most ? i : most_i;
            most = max_nan(most, v);
        }
        f.top = __shfl_sync(kFull, most, 0);
        f.top_i = __shfl_sync(kFull, most_i, 0);
        mass = times_power(mass, unit - f.unit);
        f.whole = warp_sum(mass);
        const double target = static_cast<double>(u) * f.whole, bound = EXACT ? kSlackExact : kSlackFast * f.whole;
        double start = 0.0;
        if (owner(mass, 0.0, target, lane(), &start) != rank) return f;
        const int home = owner(times_power(m, block_r - f.unit), start, target, lane(), &start);
        int tile = 0;
        double at0 = start;
        for (int k = 0; k < tiles(home); ++k) {
            const double sum = warp_sum(lane_mass<EXACT>(k, home * 32 + lane(), f.unit));
            if (!(sum > 0.0)) continue;
            tile = k;
            at0 = start;
            start += sum;
            if (start > target) break;
        }
        Tile<T> t;
        const int base = begin(home) + tile * kTileEntries;
        t.load(row, base, min(V, begin(home) + run), aligned);
        f.close = fabs(at0 - target) <= bound;
        // the entries' weights as they were added up; index order: vectors of the tile, lanes, entries of a lane
        const int own = EXACT ? 0 : static_cast<int>(s.lane_m[tile][home * 32 + lane()].y), shift = EXACT ? 0 : own - f.unit;
#pragma unroll 1
        for (int k = 0; k < Tile<T>::kVecs; ++k) {
            double e[Tile<T>::kVec], sum = 0.0;
            float v[Tile<T>::kVec];
#pragma unroll
            for (int q = 0; q < Tile<T>::kVec; ++q) {
                v[q] = t.value(q);
                e[q] = times_power(weight<EXACT>(v[q], own), shift);
                sum += e[q];
            }
            t.rotate();
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
                        mine = q;
                        z = v[q];
                        over = at > target;
                    }
                }
            }
            const unsigned any = __ballot_sync(kFull, mine >= 0), above = __ballot_sync(kFull, over);
            const int l = above ? __ffs(above) - 1 : any ? 31 - __clz(any) : -1;
            if (l >= 0) {
                f.token = base + (k * 32 + l) * Tile<T>::kVec + __shfl_sync(kFull, mine, l);
                f.tz = __shfl_sync(kFull, z, l);
            }
            if (above) break;
            at0 = __shfl_sync(kFull, at, 31);
        }
        f.close = __any_sync(kFull, f.close);
        return f;
    }
};

// log p of the row's entry `token`, whose logit is the largest, in the block that has it, by its first warp: from what the others have
// (see pick), their sums without the lane's tile, and the tile's other entries on their own.
template <typename T>
__device__ __forceinline__ double largest_logp(const Stream<T>& r, int token, double whole, int unit) {
    const int lane = threadIdx.x & 31, warp = (token - r.begin(0)) / r.run, tile = (token - r.begin(warp)) / kTileEntries;
    const int base = r.begin(warp) + tile * kTileEntries;
    Tile<T> t;
    t.load(r.row, base, min(r.V, r.begin(warp) + r.run), r.aligned);
    const float2 m = r.s.lane_m[tile][warp * 32 + lane];
    const int own = static_cast<int>(m.y), shift = own - unit;
    double others = 0.0, mine = 0.0;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        const double e = r.template weight<false>(t.value(i), own);
        if (Tile<T>::index(base, i) == token) mine = e; else others += e;
    }
    others = times_power(others, shift) + (whole - times_power(static_cast<double>(m.x), shift));
    const double logp = 0.0 - log1p(fmax(others, 0.0) / times_power(mine, shift));
    return __shfl_sync(kFull, logp, __ffs(__ballot_sync(kFull, mine > 0.0)) - 1);
}

// Rows whose rule cuts entries off.  A lane's tile is a group of 16 entries, and the pass has left the octave of its largest entry: an
// index of the row.  Where at least k groups reach an octave, at least k entries do, and all that do are in those groups.  They are
// read again, what reaches the octave goes to a list in the first block, and that block decides, with fp64 exponentials: of top-k
// and min-p all that counts is in the list.  top-p needs the mass of the others too; where that is too close, or the list does not
// reach it or has no room, the row is left to the search.  512 rows of 151936, with the launch of the search behind it: fp32 top-k 108
// us (all of it by the search 338), min-p 105 (239), top-p of a few tokens 119 (570); bf16 89 (184), 81 (143) and 95 (371).  The pass
// alone takes 87 and 62; the rest is two exchanges and the first block's end, 8 thousand clocks of a row, and blocks of the search that
// look at a row and end.  Both lists are sorted, so their order in memory, which atomics decide, changes nothing.
template <typename T>
__device__ __forceinline__ void list_row(Stream<T>& r, const SampleArgs& a, int row, const SampleRule& rule, float u, int tiles) {
    StreamShared& s = r.s;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tid = threadIdx.x;
    constexpr int kNone = -0x40000000;
    float block_top = s.warp_top[0];
#pragma unroll
    for (int i = 1; i < kWarps; ++i) block_top = max_nan(block_top, s.warp_top[i]);
    const int block_unit = static_cast<int>(r.unit_of(block_top));
    for (int k = 0; k < tiles; ++k) {
        const float2 m = s.lane_m[k][tid];
        const unsigned below = static_cast<unsigned>(block_unit - static_cast<int>(m.y));   // (a block's NaN or inf has no unit: too large)
        if (m.x > 0.f && below < kBins) atomicAdd(&s.bins[below], 1);
    }
    if (r.rank == 0 && warp == 1) s.exp2_table[lane] = exp2(lane / 32.0);
    __syncthreads();
    if (warp == 0) {
        // the octave that the block's share of the wanted number reaches
        const int valid = max(min(a.V, r.begin(kWarps)) - r.begin(0), 0);
        const int want = static_cast<int>((static_cast<long long>(valid) * (rule.top_k > 0 ? rule.top_k : kListP) + a.V - 1) / a.V);
        int n[kBins / 32], sum = 0;
#pragma unroll
        for (int q = 0; q < kBins / 32; ++q) sum += n[q] = s.bins[lane * (kBins / 32) + q];
        int upto = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(kFull, upto, o);
            if (lane >= o) upto += v;
        }
        int least = -0x7fffffff, at = upto - sum;
#pragma unroll
        for (int q = 0; q < kBins / 32; ++q) {
            at += n[q];
            if (at >= want && least == -0x7fffffff) least = block_unit - (lane * (kBins / 32) + q);
        }
        least = __reduce_max_sync(kFull, least);
        if (valid == 0 || least == -0x7fffffff) least = 0x7fffffff;   // (says nothing)
        // masses of the blocks, in units next to the largest entry
        double m = lane < kWarps ? s.warp_m[lane] : 0.0;
        const int unit = lane < kWarps && m > 0.0 ? s.warp_r[lane] : kNone, most = __reduce_max_sync(kFull, unit);
        m = warp_sum(times_power(m, unit - most));
        const int count = __reduce_add_sync(kFull, lane < kWarps ? s.warp_n[lane] : 0);
        r.expect(4 * r.ctas);
        if (lane < r.ctas) {
            send(r.box(4 * r.rank), r.mail(), lane, static_cast<unsigned long long>(__double_as_longlong(m)));
            send(r.box(4 * r.rank + 1), r.mail(), lane, static_cast<unsigned long long>(static_cast<unsigned>(most)) << 32 | static_cast<unsigned>(count));
            send(r.box(4 * r.rank + 2), r.mail(), lane, static_cast<unsigned long long>(__float_as_uint(block_top)) << 32 | static_cast<unsigned>(least));
            send(r.box(4 * r.rank + 3), r.mail(), lane, 0);
        }
        const unsigned long long* got = r.box(0);
        r.receive();
        const bool on = lane < r.ctas;
        got += 4 * (on ? lane : 0);
        double mass = on ? __longlong_as_double(static_cast<long long>(got[0])) : 0.0;
        const int their_unit = on ? static_cast<int>(got[1] >> 32) : kNone;
        float top = on ? __uint_as_float(static_cast<unsigned>(got[2] >> 32)) : -INFINITY;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(kFull, top, o));
        ListState w = {};
        w.top = top;
        w.unit = __reduce_max_sync(kFull, their_unit);
        w.whole = warp_sum(times_power(mass, their_unit - w.unit));
        w.n_all = __reduce_add_sync(kFull, on ? static_cast<int>(got[1] & 0xffffffffu) : 0);
        w.least = __reduce_min_sync(kFull, on ? static_cast<int>(got[2] & 0xffffffffu) : 0x7fffffff);
        if (w.n_all <= kList) w.least = kNone;                    // all of them
        w.floor = kLowest;
        if (rule.log_min_p > -INFINITY && top > -INFINITY && top < INFINITY) {
            w.floor = lowest_allowed(rule, top);
            const int reached = static_cast<int>(r.unit_of(w.floor));
            w.least = rule.top_k > 0 ? max(w.least, reached) : reached;
        }
        if (lane == 0) { s.known = w; s.n_listed = 0; }
    }
    __syncthreads();
    const float top = s.known.top, floor = s.known.floor;
    const int unit = s.known.unit, least = s.known.least;
    if (!(top > -INFINITY && top < INFINITY)) {                   // NaN, +inf or nothing but -inf
        if (r.rank == 0 && tid == 0) no_distribution(a, row);
        return;
    }
    // the groups that reach it; mass of the others
    unsigned marked = 0;
    double rest = 0.0;
    for (int k = 0; k < tiles; ++k) {
        const float2 m = s.lane_m[k][tid];
        if (m.x > 0.f && static_cast<int>(m.y) >= least) marked |= 1u << k;
        else rest += r.template lane_mass<false>(k, tid, unit);
    }
    const int n_marked = __popc(marked);
    int upto = n_marked;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(kFull, upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == 31) s.warp_n[warp] = upto;
    __syncthreads();                                              // from here on the masses' memory is free
    const int of_warp = lane < kWarps ? s.warp_n[lane] : 0, n_queue = __reduce_add_sync(kFull, of_warp);
    int to = upto - n_marked + __reduce_add_sync(kFull, lane < warp ? of_warp : 0);
    const bool room = n_queue <= kList && fabsf(top * r.c) <= 0x1p20f;   // (far from 0 a unit and c times a logit have no digits left to differ in)
    ListSpace& sp = s.space;
    if (room)
        for (; marked; marked &= marked - 1) sp.queue[to++] = static_cast<uint16_t>((__ffs(marked) - 1) * kThreads + tid);
    __syncthreads();
    constexpr int kVec = Tile<T>::kVec, kVecs = Tile<T>::kVecs;
    const float below = static_cast<float>(least) - 1.f;
    if (room)
        for (int i = tid; i < n_queue * kVecs; i += kThreads) {
            const int g = sp.queue[i / kVecs], t = g % kThreads, begin = r.begin(t / 32), end = min(a.V, begin + r.run);
            const int at = begin + g / kThreads * kTileEntries + i % kVecs * (32 * kVec) + t % 32 * kVec;
            float x[kVec];
            if (r.aligned && at + kVec <= end) {
#pragma unroll
                for (int q = 0; q < kVec; q += 2) { const float2 two = pair(r.row + at + q); x[q] = two.x; x[q + 1] = two.y; }
            } else {
#pragma unroll
                for (int q = 0; q < kVec; ++q) x[q] = at + q < end ? one(r.row + at + q) : -INFINITY;
            }
#pragma unroll
            for (int q = 0; q < kVec; ++q) {
                if (x[q] >= floor && fmaxf(x[q] * r.c, -1e9f) > below) {
                    const int n = atomicAdd(&s.n_listed, 1);      // (any order: they are sorted)
                    if (n < kList) sp.stage[n] = static_cast<unsigned long long>(~key_of(x[q])) << 32 | static_cast<unsigned>(at + q);
                } else {
                    rest += r.template weight<false>(x[q], unit);
                }
            }
        }
    rest = warp_sum(rest);
    if (lane == 0) s.warp_m[warp] = rest;
    __syncthreads();
    const bool by_mass = rule.top_p < 1.0 && rule.top_k == 0 && rule.log_min_p == -INFINITY;
    if (warp == 0) {
        const int n = room && s.n_listed <= kList ? s.n_listed : 2 * kList;
        rest = warp_sum(lane < kWarps ? s.warp_m[lane] : 0.0);
        r.expect(2 * r.ctas);
        if (lane < r.ctas) {
            send(r.box(4 * r.rank), r.mail(), lane, static_cast<unsigned long long>(__double_as_longlong(rest)));
            send(r.box(4 * r.rank + 1), r.mail(), lane, static_cast<unsigned>(n));
        }
        const unsigned long long* got = r.box(0);
        r.receive();
        const bool on = lane < r.ctas;
        const int theirs = on ? static_cast<int>(got[4 * lane + 1]) : 0, total = __reduce_add_sync(kFull, theirs);
        const int base = __reduce_add_sync(kFull, lane < r.rank ? theirs : 0);
        rest = warp_sum(on ? __longlong_as_double(static_cast<long long>(got[4 * lane])) : 0.0);
        if (lane == 0) {
            const bool all_there = rule.top_k == 0 || total >= min(rule.top_k, s.known.n_all) ||
                                   (rule.log_min_p > -INFINITY && least == static_cast<int>(r.unit_of(floor)));
            s.again = total > kList || !all_there || (by_mass && s.known.whole - rest < rule.top_p * s.known.whole);
            s.known.total = total;
            s.known.base = base;
            s.known.rest = rest;
        }
    }
    __syncthreads();
    r.turn = 2;
    if (s.again) {
        if (r.rank == 0 && tid == 0) a.token[row] = kUnlisted;
        return;
    }
    const int total = s.known.total, n = s.n_listed;
    if (r.rank == 0) r.expect(total);
    for (int i = tid; i < n; i += kThreads) send(&sp.list[s.known.base + i], r.mail(), 0, sp.stage[i]);
    if (r.rank != 0) return;
    if (warp == 0) r.receive();
    __syncthreads();
    // masses in units of the largest entry's
    const double others = s.known.rest * exp2(static_cast<double>(unit) - static_cast<double>(top) * static_cast<double>(r.c));
    constexpr int kEach = kList / kThreads;
    const int i0 = kEach * tid;
    r.top = top;
    // Sum over the threads before this one, and over all (`into`: a place for the warps' sums that no other sum uses).
    auto prefix = [&](double v, double* into, double* all) {
        const double run = warp_scan(v, lane);
        if (lane == 31) into[warp] = run;
        __syncthreads();
        const double w = warp_scan(lane < kWarps ? into[lane] : 0.0, lane), before = __shfl_sync(kFull, w, warp ? warp - 1 : 0);
        *all = __shfl_sync(kFull, w, kWarps - 1);
        return (warp ? before : 0.0) + (run - v);
    };
    double e[kEach], sum = 0.0, all = 0.0, listed = 0.0;
    int kept = total;
    if (rule.top_k > 0 || rule.top_p < 1.0) {
        sort_items(sp.list, total);
        const int limit = rule.top_k > 0 ? min(rule.top_k, total) : total;
#pragma unroll
        for (int h = 0; h < kEach; ++h) {
            e[h] = i0 + h < total ? r.template weight<true>(value_of(~static_cast<unsigned>(sp.list[i0 + h] >> 32)), 0) : 0.0;
            if (i0 + h < limit) sum += e[h];
        }
        const double before = prefix(sum, s.scan_a, &all);
        bool close = false;
        const double whole = by_mass ? others + all : all, target = rule.top_p * whole, bound = by_mass ? kSlackFast * whole : 0.0;
        double at = before;
        kept = 0;
#pragma unroll
        for (int h = 0; h < kEach; ++h) {
            if (i0 + h >= limit) continue;
            const bool in = rule.top_p >= 1.0 || at < target || i0 + h == 0;      // (rounding does not take the first one)
            kept += in;
            close |= by_mass && fabs(at - target) <= bound && i0 + h > 0;
            at += e[h];
        }
        kept = __reduce_add_sync(kFull, kept);
        if (lane == 0) s.warp_n[warp] = kept;
        close |= by_mass && !(all >= target + bound);
        if (__syncthreads_or(close)) {
            if (tid == 0) a.token[row] = kUnlisted;
            return;
        }
        kept = __reduce_add_sync(kFull, lane < kWarps ? s.warp_n[lane] : 0);
        // mass of the listed ones that are not kept
#pragma unroll
        for (int h = 0; h < kEach; ++h)
            if (i0 + h >= kept) listed += e[h];
        prefix(listed, s.scan_b, &listed);
    }
    // the kept ones by index
    for (int i = tid; i < kept; i += kThreads) {
        const unsigned long long item = sp.list[i];
        sp.stage[i] = item << 32 | item >> 32;
    }
    __syncthreads();
    sort_items(sp.stage, kept);
    // the largest entry stands apart: it may have nearly all of the mass
    const unsigned most = ~key_of(top);
    double others_kept = 0.0;
    sum = 0.0;
#pragma unroll
    for (int h = 0; h < kEach; ++h) {
        const unsigned key = i0 + h < kept ? static_cast<unsigned>(sp.stage[i0 + h]) : 0u;
        e[h] = i0 + h < kept ? r.template weight<true>(value_of(~key), 0) : 0.0;
        sum += e[h];
        others_kept += key == most ? 0.0 : e[h];
    }
    int tops = 0;
#pragma unroll
    for (int h = 0; h < kEach; ++h) tops += i0 + h < kept && static_cast<unsigned>(sp.stage[i0 + h]) == most;
    tops = __reduce_add_sync(kFull, tops);
    if (lane == 0) s.warp_n[warp] = tops;
    prefix(others_kept, s.scan_a, &others_kept);
    others_kept += __reduce_add_sync(kFull, lane < kWarps ? s.warp_n[lane] : 0) - 1;
    // the first one whose running mass is above the target, or, where rounding leaves none, the last with any
    double at = prefix(sum, s.scan_b, &all);
    const double want = static_cast<double>(u) * all;
    int mine = kList;
    int last = -1;
#pragma unroll
    for (int h = 0; h < kEach; ++h) {
        at += e[h];
        if (e[h] > 0.0) {
            last = i0 + h;
            if (at > want && mine == kList) mine = i0 + h;
        }
    }
    mine = __reduce_min_sync(kFull, mine);
    last = __reduce_max_sync(kFull, last);
    if (lane == 0) { s.warp_i[warp] = mine; s.warp_n[warp] = last; }
    __syncthreads();
    if (warp != 0) return;
    mine = __reduce_min_sync(kFull, lane < kWarps ? s.warp_i[lane] : kList);
    last = __reduce_max_sync(kFull, lane < kWarps ? s.warp_n[lane] : -1);
    if (lane == 0) {
        const unsigned long long item = sp.stage[mine < kList ? mine : last];
        const float z = value_of(~static_cast<unsigned>(item));
        const double x = (static_cast<double>(z) - static_cast<double>(top)) * r.inv_t;
        put_row(a, row, static_cast<int>(item >> 32), x - log1p(others + listed + others_kept), x - log1p(others_kept), kept);
    }
}

// LIST: there are rules that cut entries off.
template <typename T, bool LIST>
__global__ void __launch_bounds__(kThreads, 5) k_sample_stream(const __grid_constant__ SampleArgs a, int run, int ctas) {
    __shared__ StreamShared s;
    const int rank = ctas > 1 ? ptx::cluster_ctarank() : 0, row = blockIdx.x / ctas;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    SampleRule rule;
    float u;
    if constexpr (LIST) ptx::grid_launch_dependents();                         // the search behind it waits for its end
    if (!row_begins(a, row, rank, rule, u)) return;                            // (the same in every block of the cluster)
    if constexpr (LIST) {
        if (rule.search && !rule.list) {
            if (rank == 0 && threadIdx.x == 0) a.token[row] = kUnlisted;
            return;
        }
    } else if (rule.search) {
        return;
    }
    const T* src = static_cast<const T*>(a.logits) + row * a.ld;
    Stream<T> r{s, src, ctas, rank, run, a.V, reinterpret_cast<uintptr_t>(src) % 16 == 0, a.status, 0};
    const int begin = r.begin(warp), end = min(a.V, begin + run), tiles = r.tiles(warp);
    if (r.aligned && lane == 0 && end - begin >= 16) {
        // the whole run to L2 at once: what the registers have in flight does not cover the way to HBM
        const unsigned bytes = (end - begin) * sizeof(T) / 16 * 16;
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src + begin), "r"(bytes) : "memory");
    }
    if (threadIdx.x == 0) {
        ptx::mbar_init(&s.mail[0], 1);
        ptx::mbar_init(&s.mail[1], 1);
        ptx::fence_barrier_init();
    }
    if (LIST && threadIdx.x < kBins) s.bins[threadIdx.x] = 0;
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // the block has begun and can take messages
    const bool greedy = rule.temperature == 0.f;
    r.inv_t = rule.inv_t;
    r.c64 = 1.4426950408889634 * rule.inv_t;
    r.c = static_cast<float>(r.c64);
    // A lane's masses of its tiles, each in a unit of its own: nothing crosses lanes until all tiles are read.
    float most = -INFINITY;
    int n = 0, at_most = 0x7fffffff;
    const uint64_t c2 = ptx::pack2(r.c, r.c);
    for (int k = 0; k < tiles; ++k) {
        Tile<T> t;
        t.load(src, begin + k * kTileEntries, end, r.aligned);
        float m = max_nan(t.value(0), t.value(1)), least = fminf(t.value(0), t.value(1));
#pragma unroll
        for (int i = 2; i < kPerLane; i += 2) {
            m = max_nan(m, t.value(i), t.value(i + 1));
            least = min3(least, t.value(i), t.value(i + 1));
        }
        n += kPerLane;
        if (least == -INFINITY)
#pragma unroll
            for (int i = 0; i < kPerLane; ++i) n -= t.value(i) == -INFINITY;
        if (greedy && m > most) {
#pragma unroll
            for (int i = kPerLane - 1; i >= 0; --i) at_most = t.value(i) == m ? Tile<T>::index(begin + k * kTileEntries, i) : at_most;
        }
        most = max_nan(most, m);
        const float unit = r.unit_of(m);
        const uint64_t u2 = ptx::pack2(-unit, -unit);
        uint64_t e2[kPerLane / 2];
#pragma unroll
        for (int i = 0; i < kPerLane / 2; ++i) {
            float x, y;
            ptx::unpack2(ptx::fma2(ptx::pack2(t.value(2 * i), t.value(2 * i + 1)), c2, u2), x, y);
            e2[i] = ptx::pack2(ptx::ex2(x), ptx::ex2(y));
        }
#pragma unroll
        for (int o = kPerLane / 4; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < o; ++i) e2[i] = ptx::add2(e2[i], e2[i + o]);
        float x, y;
        ptx::unpack2(e2[0], x, y);
        s.lane_m[k][threadIdx.x] = make_float2(x + y, unit);
    }
    // the warp's mass, in a unit next to its largest entry
    const int unit = __reduce_max_sync(kFull, static_cast<int>(r.unit_of(most)));
    double mass = 0.0;
    for (int k = 0; k < tiles; ++k) mass += r.template lane_mass<false>(k, threadIdx.x, unit);
    mass = warp_sum(mass);
    float top = most;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(kFull, top, o));
    const int top_i = __reduce_min_sync(kFull, most == top ? at_most : 0x7fffffff);   // (greedy's)
    n = __reduce_add_sync(kFull, n);
    if (lane == 0) {
        s.warp_m[warp] = mass;
        s.warp_r[warp] = unit;
        s.warp_top[warp] = top;
        s.warp_i[warp] = top_i;
        s.warp_n[warp] = n;
    }
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");        // before the first message
    __syncthreads();
    if constexpr (LIST) {
        if (rule.search) {
            list_row(r, a, row, rule, u, tiles);
            return;
        }
    }
    if (warp == 0) {
        const auto f = r.template locate<false>(u);
        int again = 0;
        if (!(f.top > -INFINITY && f.top < INFINITY)) {              // NaN, +inf or nothing but -inf
            if (rank == 0 && lane == 0) no_distribution(a, row);
        } else {
            // log of the whole mass: its unit, less what the rounding of c adds to every exponent alike
            const double lse = (log2(f.whole) + f.unit - static_cast<double>(f.top) * (static_cast<double>(r.c) - r.c64)) * 0.69314718055994531;
            const bool fits = fabsf(f.top * r.c) <= 0x1p20f;          // (far from 0 a unit and c times a logit have no digits left to differ in)
            if (greedy) {
                again = !fits;                                       // (the same in every block)
                if (fits && f.top_i / (kWarps * run) == rank) {
                    const double logp = largest_logp(r, f.top_i, f.whole, f.unit);
                    if (lane == 0) put_row(a, row, f.top_i, logp, 0.0, 1);
                }
            } else {
                r.expect(ctas);
                if (lane < ctas) send(r.box(rank), r.mail(), lane, f.close || !fits);
                const unsigned long long* got = r.box(0);
                r.receive();
                again = __any_sync(kFull, lane < ctas && got[lane < ctas ? lane : 0] != 0);
                if (!again && f.token >= 0) {
                    const double logp = f.tz == f.top ? largest_logp(r, f.token, f.whole, f.unit) : static_cast<double>(f.tz) * rule.inv_t - lse;
                    if (lane == 0) put_row(a, row, f.token, logp, logp, f.n);
                }
            }
        }
        if (lane == 0) { s.again = again; s.top = f.top; }
    }
    __syncthreads();
    if (!s.again) return;
    r.top = s.top;
    if (warp == 0) s.exp2_table[lane] = exp2(lane / 32.0);
    __syncthreads();
    mass = 0.0;
    for (int k = 0; k < tiles; ++k) {
        Tile<T> t;
        t.load(src, begin + k * kTileEntries, end, r.aligned);
        double m = 0.0;
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) m += r.template weight<true>(t.value(i), 0);
        s.lane_x[k][threadIdx.x] = m;
        mass += m;
    }
    mass = warp_sum(mass);
    if (lane == 0) { s.warp_m[warp] = mass; s.warp_r[warp] = 0; }
    __syncthreads();
    if (warp != 0) return;
    const auto f = r.template locate<true>(u);
    if (greedy) {
        if (f.top_i / (kWarps * run) == rank && lane == 0) put_row(a, row, f.top_i, 0.0 - log(f.whole), 0.0, 1);
    } else if (f.token >= 0 && lane == 0) {
        const double logp = (static_cast<double>(f.tz) - static_cast<double>(f.top)) * rule.inv_t - log(f.whole);
        put_row(a, row, f.token, logp, logp, f.n);
    }
}

// The search's entries of a thread with so many blocks per row.  They are read in pairs, and the threads' first ones lie an odd number of
// pairs apart: at different banks.
constexpr int entries_of_thread(int V, int ctas) { return (((V + kThreads * ctas - 1) / (kThreads * ctas) + 1) / 2 | 1) * 2; }
constexpr int kSearchBytes = 40 * 1024;      // of a block where fewer than 16 share the row
// The most that a block of the search asks for.
constexpr int kMaxSearchBytes = std::max<int>(entries_of_thread(UNITY_MAX_SAMPLE_V, kMaxCluster) * kThreads * sizeof(float), kSearchBytes);

template <typename... P, typename... A>
cudaError_t launch_clusters(void (*kernel)(P...), int rows, int ctas, int bytes, bool early, cudaStream_t st, const A&... args) {
    // The limit belongs to the function, whichever contexts and host threads launch it: always that of the largest call, so that no call
    // takes away what another is about to use.
    cudaError_t e = bytes > 0 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSearchBytes) : cudaSuccess;
    if (e == cudaSuccess && ctas > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(rows) * ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = early ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, bool bf16, bool any_search, bool any_list, bool any_other, int sm_count, cudaStream_t st, int* n_launches) {
    // The search: the fewest blocks per row (1 .. 16) whose share takes at most 40 KB, so that four blocks fit an SM; more while the rows
    // leave some without one.
    const int width = bf16 ? 2 : 4;
    int search_ctas = 1, per = 0;
    for (;; search_ctas *= 2) {
        per = entries_of_thread(a.V, search_ctas);
        if (search_ctas == kMaxCluster) break;
        if (static_cast<long long>(per) * kThreads * width <= kSearchBytes && (per <= 16 || static_cast<long long>(a.n_rows) * search_ctas >= 4 * sm_count)) break;
    }
    // With room for all rows at once the search alone takes less than a pass and then the search's launch (top-k of 151936 fp32, 1 / 8
    // / 32 / 64 rows: 15 / 19 / 33 / 52 us against 20 / 23 / 31 / 27).
    const bool list = any_list && static_cast<long long>(a.n_rows) * search_ctas > 4 * sm_count;
    if (list || any_other) {
        // A warp's run of entries: up to 20 tiles.  More blocks per row while a run is longer than a tile and the rows do not fill the
        // machine several times over: a block ends with a phase of one warp, which others have to cover (512 rows of 151936, 2 / 4 / 8 / 16
        // blocks per row: fp32 99 / 90 / 85 / 130 us, bf16 63 / 60 / 76 / 128 us).
        // With lists a row ends with more than that: runs of up to 20 KB, and two blocks per SM are enough (top-k with top-p,
        // blocks per row: 512 rows fp32 122 / 110 / 118 us at 2 / 4 / 8, 128 rows fp32 43 / 47 / 60 at 4 / 8 / 16, bf16 35 / 42 / 61).
        const long long enough = (list ? 2LL : bf16 ? 8LL : 16LL) * sm_count;
        const int longest = list ? std::min(kMaxTiles * kTileEntries, 20 * 1024 / width) : kMaxTiles * kTileEntries;
        int ctas = 1, run = 0;
        for (;; ctas *= 2) {
            run = ((a.V + kWarps * ctas - 1) / (kWarps * ctas) + 7) / 8 * 8;
            if (ctas == kMaxCluster) break;
            if (run <= longest && (run <= kTileEntries || static_cast<long long>(a.n_rows) * ctas >= enough)) break;
        }
        const cudaError_t e = launch_clusters(list ? bf16 ? k_sample_stream<__nv_bfloat16, true> : k_sample_stream<float, true>
                                                   : bf16 ? k_sample_stream<__nv_bfloat16, false> : k_sample_stream<float, false>,
                                              a.n_rows, ctas, 0, false, st, a, run, ctas);
        if (e != cudaSuccess) return e;
        *n_launches += 1;
    }
    if (any_search) {
        const cudaError_t e = launch_clusters(bf16 ? k_sample<__nv_bfloat16> : k_sample<float>, a.n_rows, search_ctas, per * kThreads * width, list, st, a, per,
                                              search_ctas, list ? 1 : 0);
        if (e != cudaSuccess) return e;
        *n_launches += 1;
    }
    return cudaSuccess;
}

}  // namespace unity
