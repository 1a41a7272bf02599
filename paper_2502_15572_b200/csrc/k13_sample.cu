// K13 -- verification of drafts against the model's distribution, from given random numbers (no drafts: sampling).
//
// A sequence is a chain: the token drawn at depth t decides which row of logits is read at depth t + 1, so that only the rows on
// the path are read, at most L + 1 of the 1 + n L.  One cluster follows a sequence; its CTAs share a row by contiguous pieces, which
// they keep in shared memory as far as it goes.  Per row: the maximum; the cuts of top_k and top_p; the weights' sums piece by piece; and
// the piece, warp, lane and element where the running sum passes u times the whole.  Bytes are not what a row costs.  32000 16-bit logits in 16 CTAs, top_p, the second row
// of a sequence and later ones, cycles by the SM's clock at one thread (24600 in all; each step's wait for slower warps and CTAs is part of the next one):
//     reading and the CTA's maximum 1000, its exchange 1400; first histogram 4300, its search 6400 (with the wait for the slowest
//     CTA's histogram); second one 1400, 2500; pass for the running sums 1900, their sums in the CTA 900, exchange 1400; search for the token 1000, last exchange 2000;
//     the next row's choice 400.  Without top_p 11400.
// Instructions come from far at the first depth (30000 cycles; 45000 in a process's first call), so loops are not unrolled where that multiplies long code (32000 logits, top_p: 22.0 us a row so, 18.8 us without).
//
// A weight is rint(2^42 e^((x - max) / T)), a whole number: sums are exact, so they depend neither on their order nor on how
// many CTAs share a row, and a token is the same whatever the batch.
//
// Cuts are found from the largest logit down with histograms of 2048 bins.  The first one has bins of equal width in (max - x) / T, over the 44 octaves in
// which weights are not 0: logits spread over many of them, while bits of a float's exponent would put most into a few, whose
// atomic additions then wait for one another.  Further ones divide the range of keys of the bin that was hit, until a bin is one key; the
// second one is the last for 16-bit logits as a rule, and looks at one group of 32 bins.  A small top_k needs none of this: see few().
//
// Measured (device): one row of 32000 with top_p 18 us, with top_k 50 12.5; ten drafts of ten of 32000 29.6; 16 sequences of 3 x 20 of 100003 77 (some 8600
// cycles a row); 64 rows of 151001 in fp32, normal logits: greedy 27.8, temperature alone 49, top_k 40 25.5 (1.5 TB/s: reading, then one exchange after the other), top_k 200 70, with
// top_p 110, top_p alone 103 (spread 4, temperature 0.7) to 120 (2, 1): whole rows are gone through three times, their weights computed twice.
#include <atomic>
#include <cfloat>

#include "common.cuh"
#include "internal.h"

namespace dresd {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kMaxCtas = 16;
constexpr int kBins = 2048, kGroups = kBins / 32, kSteps = 64;
constexpr int kFew = 512, kFewKept = 128;                     // see few()
constexpr double kOne = 4398046511104.0;                       // 2^42, the largest weight
constexpr float kOctaves = 44.f;                               // a weight 2^-44 of the largest rounds to 0
constexpr int kTable = 64;                                     // 2^(-j / 64)

typedef unsigned long long u64;

template <typename T> struct Logit;
template <> struct Logit<float> {
    static constexpr uint32_t kLowest = 0xFF800000u;           // -infinity
    static constexpr int kGrain = 0;                           // low bits of float_to_ordered() that are the same for all
    static __device__ __forceinline__ float value(float x) { return x; }
};
template <> struct Logit<__half> {
    static constexpr uint32_t kLowest = 0xFC00FC00u;
    static constexpr int kGrain = 13;
    static __device__ __forceinline__ float value(__half x) { return __half2float(x); }
};
template <> struct Logit<__nv_bfloat16> {
    static constexpr uint32_t kLowest = 0xFF80FF80u;
    static constexpr int kGrain = 16;
    static __device__ __forceinline__ float value(__nv_bfloat16 x) { return __bfloat162float(x); }
};

// A row of logits at any address, as blocks of 16 bytes from the boundary at or before its first element.
template <typename T> struct Row {
    static constexpr int kVec = 16 / sizeof(T);
    const T *base;               // of block 0; elements outside first .. last - 1 are not the row's
    int first, last, blocks;
    __device__ __forceinline__ Row(const T *row, int V)
    {
        first = (int)(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T));
        base = row - first;
        last = first + V;
        blocks = (last + kVec - 1) / kVec;
    }
    // Block q; what is not the row's is -infinity.
    __device__ __forceinline__ uint4 load(int q) const
    {
        const int j = q * kVec;
        if (j >= first && j + kVec <= last) return __ldg(reinterpret_cast<const uint4 *>(base + j));
        constexpr uint32_t low = Logit<T>::kLowest;
        uint4 w = make_uint4(low, low, low, low);
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (j + i >= first && j + i < last) reinterpret_cast<T *>(&w)[i] = base[j + i];
        return w;
    }
};
template <typename T> __device__ __forceinline__ void values(const uint4 &w, float (&x)[16 / sizeof(T)])
{
#pragma unroll
    for (int i = 0; i < (int)(16 / sizeof(T)); ++i) x[i] = Logit<T>::value(reinterpret_cast<const T *>(&w)[i]);
}

// What remains of a row: logits that are larger than x, and the first `ties` of those that are equal.  NaN is neither.
struct Cut {
    float x;
    int ties;
};

struct alignas(16) Shared {                     // the cache of 16-byte blocks lies behind it
    u64 bins[2][kBins];                        // the halves are added to apart.  Two: the one before is read by the other CTAs until the next barrier
    u64 group[2][kMaxCtas][kGroups];           // of 32 bins each, of every CTA of the cluster
    u64 weight[kWarps][kSteps];                // of a warp's consecutive blocks, and its logits that are tied
    int ties[kWarps][kSteps];
    long long table[kTable];                   // 2^62 2^(-j / 64)
    double rate;                               // log2(e) / T, the sequence's, and what follows from it
    float rate_high, rate_low, span, bin_rate;
    double log_whole;
    u64 warp_weight[kWarps];
    int warp_ties[kWarps], warp_count[kWarps];
    uint32_t warp_top[kWarps];
    u64 total[kMaxCtas];                       // of every CTA; likewise the next three
    int tied[kMaxCtas];
    int count[kMaxCtas];                       // of logits above -infinity
    uint32_t top[kMaxCtas];
    float2 few[kFew];                          // of the cluster's first CTA: logits that are left, with the bits of their indices, in any order
    float2 kept[kFewKept];                     // the largest of them, in order
    u64 kept_weight[2][kFewKept];              // without and with top_p
    int few_count;
    u64 above, target;                         // found by warp 0
    int position;
    int token;                                 // written by the CTA that finds it, in every CTA
    float logit;
};
static_assert(sizeof(Shared) % 16 == 0, "blocks behind it are aligned");

template <typename V> __device__ __forceinline__ V *in_cta(V *p, uint32_t rank)
{
    u64 r;
    asm("mapa.u64 %0, %1, %2;" : "=l"(r) : "l"(reinterpret_cast<u64>(p)), "r"(rank));
    return reinterpret_cast<V *>(r);
}

__device__ __forceinline__ u64 sum_warp(u64 x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}
// Inclusive sums over the lanes.
template <typename V> __device__ __forceinline__ V scan_warp(V x)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V y = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if (lane >= o) x += y;
    }
    return x;
}

template <typename T>
struct Sampler {
    static constexpr int kVec = Row<T>::kVec;
    Shared &s;
    uint4 *const cache;          // this CTA's first blocks in shared memory
    const int cached;
    const uint32_t rank, ctas;
    const Row<T> row;
    int q0, q1;                  // this CTA's blocks
    float top, least;            // the row's largest logit; a logit that is not above `least` has no weight
    float rate, rate_low;        // log2(e) / T
    float top_high, top_low;     // top log2(e) / T, the first part a multiple of 1/64 and not less
    float bin_rate;              // half logits to bins
    int buffer;                  // histogram that is free
    int w0, w1;                  // this warp's blocks
    __device__ __forceinline__ Sampler(Shared &s_, uint4 *cache_, int cached_, uint32_t rank_, uint32_t ctas_, const T *p, int V)
        : s(s_), cache(cache_), cached(cached_), rank(rank_), ctas(ctas_), row(p, V), buffer(0)
    {
        const int per = (row.blocks + ctas - 1) / ctas;
        q0 = min((int)rank * per, row.blocks);
        q1 = min(q0 + per, row.blocks);
        const int each = (q1 - q0 + kWarps - 1) / kWarps;
        w0 = min(q0 + (int)(threadIdx.x >> 5) * each, q1);
        w1 = min(w0 + each, q1);
    }
    __device__ __forceinline__ void block(int q, float (&x)[kVec]) const { values<T>(q - q0 < cached ? cache[q - q0] : row.load(q), x); }

    // What weight() and bin() need of the temperature (one thread, once: fp64) and of the maximum.
    static __device__ __forceinline__ void set_rate(Shared &s, double r)
    {
        s.rate = r;
        s.rate_high = (float)r;
        s.rate_low = (float)(r - (double)s.rate_high);
        s.span = (float)((double)kOctaves / r);
        s.bin_rate = fminf((float)(2. * r * (kBins / (double)kOctaves)), 1e38f);
    }
    __device__ __forceinline__ void scales()
    {
        rate = s.rate_high;
        rate_low = s.rate_low;
        bin_rate = s.bin_rate;
        const float t = __fmul_rn(top, rate);
        top_high = ceilf(t * (float)kTable) * (1.f / kTable);
        top_low = __fadd_rn(__fsub_rn(t, top_high), __fmaf_rn(top, rate_low, __fmaf_rn(top, rate, -t)));
        least = fmaxf(top - s.span, -FLT_MAX);
        if (!(least < top)) least = nextafterf(top, -INFINITY);
    }
    // 2^42 2^-y, y = (top - x) log2(e) / T, as a whole number: k = rint(64 y), 2^(-k / 64) is a power of two times a table's entry (Tang 1989),
    // and 2^-r, r = y - k / 64, five terms of its series.  fp64 has an eighth of fp32's rate here, so r is computed as
    // (top_high - k / 64 - x rate) + (top_low - x rate_low), whose first difference is exact and whose fma is rounded when what
    // is large has gone: off by 2^-28 at most, relative to the weight.  That needs |top| log2(e) / T < 2^12; beyond (kWide), x - top comes first, as a sum of two
    // floats (Knuth).  No branch: the chain is long, and a thread has several logits to do at once.
    template <bool kWide> __device__ __forceinline__ u64 weight_by(float x) const
    {
        constexpr float kRound = 12582912.f;                                // 1.5 2^23: the sum's low bits are the nearest whole number
        float near, r;
        if constexpr (!kWide) {
            near = __fmaf_rn(x, -(float)kTable * rate, __fmaf_rn(top_high, (float)kTable, kRound));
            const float rest = __fmaf_rn(__fsub_rn(near, kRound), -1.f / kTable, top_high);       // exact
            r = __fadd_rn(__fmaf_rn(-x, rate, rest), __fmaf_rn(-x, rate_low, top_low));
        } else {
            const float d = __fsub_rn(top, x), back = __fsub_rn(d, top);
            const float d_low = __fsub_rn(__fsub_rn(top, __fsub_rn(d, back)), __fadd_rn(x, back));
            const float y = __fmul_rn(d, rate);
            near = __fmaf_rn(y, (float)kTable, kRound);
            const float low = __fmaf_rn(d_low, rate, __fmaf_rn(d, rate_low, __fmaf_rn(d, rate, -y)));
            r = __fadd_rn(__fmaf_rn(__fsub_rn(near, kRound), -1.f / kTable, y), low);
        }
        const int k = __float_as_int(near) - 0x4B400000;
        constexpr float a = 0.6931471805599453f;
        // (2^-r - 1) 2^32
        const float e = __fmul_rn(r, __fmaf_rn(r, __fmaf_rn(r, __fmaf_rn(r, a * a * a * a / 24.f * 0x1p32f, a * a * a / -6.f * 0x1p32f), a * a / 2.f * 0x1p32f), -a * 0x1p32f));
        const long long entry = s.table[k & (kTable - 1)];
        const u64 w = (u64)(entry + (long long)(int)(entry >> 32) * __float2int_rn(e));
        const u64 v = ((w >> 19 >> (k >> 6 & 63)) + 1) >> 1;
        return x == top ? (u64)kOne : x > least ? v : 0;
    }
    __device__ __forceinline__ bool wide() const { return fabsf(top_high) >= 4096.f; }
    __device__ __forceinline__ u64 weight(float x) const { return wide() ? weight_by<true>(x) : weight_by<false>(x); }
    __device__ __forceinline__ void weights(const float (&x)[kVec], u64 (&w)[kVec]) const
    {
        if (!wide()) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) w[i] = weight_by<false>(x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) w[i] = weight_by<true>(x[i]);
        }
    }
    // Weights above the cut and logits at it, of a block; all lanes of a warp together.
    __device__ __forceinline__ void sums(const float (&x)[kVec], const Cut &cut, u64 &w, int &n) const
    {
        bool any = false;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            any |= x[i] > cut.x && x[i] > least;
            n += x[i] == cut.x;
        }
        if (!__any_sync(0xFFFFFFFFu, any)) return;
        u64 v[kVec];
        weights(x, v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) w += x[i] > cut.x ? v[i] : 0;
    }
    // Bin of equal widths, from the largest logit down; it does not fall where x falls.  (Halves: no overflow.)
    __device__ __forceinline__ int bin(float x) const
    {
        return x == top ? 0 : (int)fminf((0.5f * top - 0.5f * x) * bin_rate, (float)(kBins - 1));
    }
    // A number that no logit of bins 0 .. b is below, but few of the others: the edge, moved by more than the roundings of bin().
    __device__ __forceinline__ float edge(int b) const
    {
        if (b >= kBins - 1 || !(bin_rate > 0.f) || !(top < INFINITY)) return -FLT_MAX;
        return fmaxf(__double2float_rd((double)top - (b + 1) * (2. / (double)bin_rate * (1. + 0x1p-20))), -FLT_MAX);
    }
    static __device__ __forceinline__ uint32_t key(float x) { return float_to_ordered(x + 0.f) >> Logit<T>::kGrain; }
    static __device__ __forceinline__ float of_key(uint32_t k)
    {
        constexpr int low = Logit<T>::kGrain;
        const uint32_t u = k << low;
        return ordered_to_float(u & 0x80000000u ? u : u | ((1u << low) - 1));
    }

    // The row's largest logit and how many logits there are above -infinity.  Fills the cache; `mine`: the thread's largest.  first: the
    // sequence's first row, nothing has been sent to another CTA yet.
    __device__ __forceinline__ int maximum(float &mine, bool first)
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        float m = -INFINITY;
        int n = 0;
#pragma unroll 4
        for (int q = q0 + threadIdx.x; q < q1; q += kThreads) {
            const uint4 w = row.load(q);
            if (q - q0 < cached) cache[q - q0] = w;
            float x[kVec];
            values<T>(w, x);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                m = fmaxf(m, x[i]);
                n += x[i] > -INFINITY;
            }
        }
        mine = m;
        n = __reduce_add_sync(0xFFFFFFFFu, n);
        uint32_t k = __reduce_max_sync(0xFFFFFFFFu, float_to_ordered(m + 0.f));
        if (lane == 0) {
            s.warp_count[warp] = n;
            s.warp_top[warp] = k;
        }
        __syncthreads();
        if (first) cluster_wait();                            // every CTA has begun: its shared memory may be written
        if (warp == 0) {
            n = __reduce_add_sync(0xFFFFFFFFu, lane < kWarps ? s.warp_count[lane] : 0);
            k = __reduce_max_sync(0xFFFFFFFFu, lane < kWarps ? s.warp_top[lane] : 0u);
            if (lane < (int)ctas) {
                *in_cta(&s.count[rank], lane) = n;
                *in_cta(&s.top[rank], lane) = k;
            }
        }
        cluster_sync_all();
        const bool there = lane < (int)ctas;
        n = __reduce_add_sync(0xFFFFFFFFu, there ? s.count[lane] : 0);
        top = ordered_to_float(__reduce_max_sync(0xFFFFFFFFu, there ? s.top[lane] : 0u));
        return n;
    }

    // Frees a histogram; by the threads from `from` on.
    __device__ __forceinline__ void clear(int which, int from)
    {
        uint4 *bins = reinterpret_cast<uint4 *>(s.bins[which]);
        for (int i = (int)threadIdx.x - from; i < kBins / 2; i += kThreads - from) bins[i] = make_uint4(0, 0, 0, 0);
    }
    // Adds `v` to positions at[i] >= 0 of the free histogram.  The low halves first, all of them on their way before a carry is looked at.
    template <bool by_weight, int kCount> __device__ __forceinline__ void add(const int (&at)[kCount], const u64 (&v)[kCount])
    {
        uint32_t old[kCount];
#pragma unroll
        for (int i = 0; i < kCount; ++i)
            if (at[i] >= 0) old[i] = atomicAdd(reinterpret_cast<uint32_t *>(s.bins[buffer] + at[i]), (uint32_t)v[i]);
        if (by_weight) {
#pragma unroll
            for (int i = 0; i < kCount; ++i) {
                const uint32_t hi = (uint32_t)(v[i] >> 32) + (old[i] + (uint32_t)v[i] < old[i] ? 1u : 0u);
                if (at[i] >= 0 && hi) atomicAdd(reinterpret_cast<uint32_t *>(s.bins[buffer] + at[i]) + 1, hi);
            }
        }
    }
    template <bool by_weight> __device__ __forceinline__ void add_one(int at, u64 v)
    {
        const int where[1] = {at};
        const u64 what[1] = {v};
        add<by_weight, 1>(where, what);
    }
    // The first position of the cluster's histogram whose running sum, `before` included, reaches `target`; what lies before it replaces `before`.
    // positions: a multiple of 32.  share >= 0: the target is that share of all.  Frees the other histogram.
    __device__ __forceinline__ int find(int positions, u64 &before, u64 &target, float share)
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        __syncthreads();
        if (positions > 32) {
            // four threads a group; each has the sum and sends it to a quarter of the cluster
            static_assert(kThreads == 4 * kGroups, "four threads a group");
            const ulonglong2 *mine = reinterpret_cast<const ulonglong2 *>(s.bins[buffer] + threadIdx.x * 8);
            u64 v = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) v += mine[i].x + mine[i].y;
            v += __shfl_xor_sync(0xFFFFFFFFu, v, 1);
            v += __shfl_xor_sync(0xFFFFFFFFu, v, 2);
            for (uint32_t c = threadIdx.x & 3; c < ctas; c += 4) *in_cta(&s.group[buffer][rank][threadIdx.x >> 2], c) = v;
        }
        cluster_sync_all();
        if (warp == 0) {                                  // of every CTA, alike
            u64 at = before;
            int g = 0;
            if (positions > 32) {
                u64 a = 0, b = 0;
#pragma unroll
                for (uint32_t c = 0; c < kMaxCtas; ++c) {
                    const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(&s.group[buffer][c][2 * lane]);
                    a += c < ctas ? v.x : 0;
                    b += c < ctas ? v.y : 0;
                }
                const u64 up_to = scan_warp(a + b);
                if (share >= 0.f) {
                    const u64 all = __shfl_sync(0xFFFFFFFFu, up_to, 31);
                    target = max((u64)__double2ll_ru((double)share * (double)all), 1ull);
                }
                const unsigned m = __ballot_sync(0xFFFFFFFFu, at + up_to >= target);
                const int l = m ? __ffs(m) - 1 : 31;
                at += __shfl_sync(0xFFFFFFFFu, up_to - a - b, l);
                const u64 one = __shfl_sync(0xFFFFFFFFu, a, l);
                g = 2 * l;
                if (at + one < target) {
                    at += one;
                    ++g;
                }
            }
            u64 v = 0, y[kMaxCtas];
#pragma unroll
            for (uint32_t c = 0; c < kMaxCtas; ++c) y[c] = *in_cta(&s.bins[buffer][g * 32 + lane], min(c, ctas - 1));   // all on their way at once
#pragma unroll
            for (uint32_t c = 0; c < kMaxCtas; ++c) v += c < ctas ? y[c] : 0;
            const u64 run = scan_warp(v);
            const unsigned m = __ballot_sync(0xFFFFFFFFu, at + run >= target);
            const int l = m ? __ffs(m) - 1 : 31;
            at += __shfl_sync(0xFFFFFFFFu, run - v, l);
            if (lane == 0) {
                s.position = g * 32 + l;
                s.above = at;
                s.target = target;
            }
        } else {
            clear(buffer ^ 1, 32);                        // nobody reads the last one any more
        }
        __syncthreads();
        before = s.above;
        target = s.target;
        buffer ^= 1;
        return s.position;
    }
    // f(x) for blocks from .. to - 1 in turn, `stride` at a time, the next load ahead; f is called by whole warps (what is not there is
    // -infinity).  One copy of f: at depth 0 its instructions come from far.
    template <typename F> __device__ __forceinline__ void each_block(int from, int to, int stride, F &&f) const
    {
        const int me = stride == 32 ? threadIdx.x & 31 : threadIdx.x;
        auto load = [&](int q) {
            constexpr uint32_t low = Logit<T>::kLowest;
            return q >= to ? make_uint4(low, low, low, low) : q - q0 < cached ? cache[q - q0] : row.load(q);
        };
        const int steps = to > from ? (to - from + stride - 1) / stride : 0;
        uint4 next = load(from + me);
#pragma unroll 1
        for (int j = 0; j < steps; ++j) {
            float x[kVec];
            values<T>(next, x);
            next = load(from + (j + 1) * stride + me);
            f(x, j);
        }
    }

    // A small top_k (of fewer logits than there are): the token from the k largest logits themselves.  The k-th largest of the threads' largest logits
    // is not above the k-th largest of all, so only threads whose largest (`mine`) is not below it have to look at theirs again; what they
    // find is brought to the first CTA.  There a logit's place in the order, and its running sums, are counted against each of the others.
    // Nothing depends on the order in which they came.  false: more than kFew of them, nothing is drawn.
    // (64 rows of 151001, top_k 40, top_p: 25.5 us; with histograms of what is left in lists 48.7, of whole rows 103.)
    __device__ __forceinline__ bool few(int k, float p, float u, float mine, float &logit, int &token)
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        if (mine > -INFINITY) add_one<false>(bin(mine), 1);
        u64 none = 0, aim = k;
        const float low = edge(find(kBins, none, aim, -1.f));
        int *const count = in_cta(&s.few_count, 0);
        float2 *const found = in_cta(s.few, 0);
        for (unsigned m = __ballot_sync(0xFFFFFFFFu, mine >= low); m; m &= m - 1) {
            // the warp looks at that thread's blocks
            const int first = q0 + warp * 32 + __ffs(m) - 1;
            for (int q = first + lane * kThreads; q < q1; q += 32 * kThreads) {
                float x[kVec];
                block(q, x);
#pragma unroll
                for (int i = 0; i < kVec; ++i)
                    if (x[i] >= low) {
                        const int at = atomicAdd(count, 1);
                        if (at < kFew) found[at] = make_float2(x[i], __int_as_float(q * kVec + i - row.first));
                    }
            }
        }
        cluster_sync_all();
        const int all = *count;
        if (all > kFew) {
            cluster_sync_all();                                   // before the count is set back
            return false;
        }
        if (rank == 0) {
            for (int i = threadIdx.x; i < all; i += kThreads) {
                const float2 me = s.few[i];
                int before = 0;
                for (int j = 0; j < all; ++j) {
                    const float2 other = s.few[j];
                    before += other.x > me.x || (other.x == me.x && __float_as_int(other.y) < __float_as_int(me.y));
                }
                if (before < k) {
                    s.kept[before] = me;
                    s.kept_weight[0][before] = weight(me.x);
                }
            }
            __syncthreads();
            const int r = threadIdx.x;
            if (r < k) {
                u64 before = 0, whole = 0;
                for (int j = 0; j < k; ++j) {
                    const u64 w = s.kept_weight[0][j];
                    whole += w;
                    before += j < r ? w : 0;
                }
                const u64 target = p < 1.f ? max((u64)__double2ll_ru((double)fmaxf(p, 0.f) * (double)whole), 1ull) : ~0ull;
                s.kept_weight[1][r] = before < target ? s.kept_weight[0][r] : 0;
            }
            __syncthreads();
            if (r < k || r == kFewKept) {
                const int me = r < k ? __float_as_int(s.kept[r].y) : 0;
                u64 before = 0, whole = 0;
                for (int j = 0; j < k; ++j) {
                    const u64 w = s.kept_weight[1][j];
                    whole += w;
                    before += __float_as_int(s.kept[j].y) < me ? w : 0;
                }
                if (r == kFewKept) {
                    s.log_whole = ::log((double)whole / kOne);    // by a warp of its own
                } else {
                    const u64 at = target_of(u, whole);
                    if (before <= at && at < before + s.kept_weight[1][r])
                        for (uint32_t c = 0; c < ctas; ++c) {
                            *in_cta(&s.token, c) = me;
                            *in_cta(&s.logit, c) = s.kept[r].x;
                        }
                }
            }
        }
        cluster_sync_all();
        logit = s.logit;
        token = s.token;
        return true;
    }
    // floor(u S)
    static __device__ __forceinline__ u64 target_of(float u, u64 whole)
    {
        return (u64)__double2ll_rz((double)fminf(fmaxf(u, 0.f), 1.f - 0x1p-24f) * (double)whole);
    }

    // The shortest part of `cut`, in descending order and then by index, whose weights reach the share `p` of all its weights (by weight), or that
    // has `k` logits (otherwise; it has more in all).
    template <bool by_weight>
    __device__ __forceinline__ Cut select(const Cut &cut, float p, u64 k)
    {
        u64 before = 0, target = k;
        const float low = by_weight ? least : -FLT_MAX;       // logits below are not looked at
        // the first histogram
        each_block(q0, q1, kThreads, [&](const float (&x)[kVec], int) {
            bool any = false;
#pragma unroll
            for (int i = 0; i < kVec; ++i) any |= x[i] > cut.x && x[i] >= low;
            if (!__any_sync(0xFFFFFFFFu, any)) return;
            u64 v[kVec];
            int at[kVec];
            if (by_weight) weights(x, v);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                if (!by_weight) v[i] = 1;
                at[i] = x[i] > cut.x && x[i] >= low && v[i] > 0 ? bin(x[i]) : -1;
            }
            add<by_weight, kVec>(at, v);
        });
        const bool first = rank == 0 && threadIdx.x == 0;
        if (first && cut.ties > 0) add_one<by_weight>(bin(cut.x), (u64)cut.ties * (by_weight ? weight(cut.x) : 1));
        const int hit = find(kBins, before, target, by_weight ? p : -1.f);
        // keys that the bin can have, and a few more
        float most = top, bottom = edge(hit);
        if (hit > 0 && bin_rate > 0.f && top < INFINITY)
            most = fminf(top, __double2float_ru((double)top - hit * (2. / (double)bin_rate * (1. - 0x1p-20))));
        while (true) {
            const uint32_t hi = key(most), lo = key(bottom);
            const int shift = max(32 - __clz(hi - lo) - 11, 0);
            each_block(q0, q1, kThreads, [&](const float (&x)[kVec], int) {
                bool any = false;
#pragma unroll
                for (int i = 0; i < kVec; ++i) any |= x[i] > cut.x && x[i] >= bottom && x[i] <= most;
                if (!__any_sync(0xFFFFFFFFu, any)) return;
                unsigned few = 0;
#pragma unroll
                for (int i = 0; i < kVec; ++i) few |= x[i] > cut.x && x[i] >= bottom && x[i] <= most ? 1u << i : 0u;
#pragma unroll 1
                for (; few; few &= few - 1) {
                    float one = x[0];
#pragma unroll
                    for (int i = 1; i < kVec; ++i) one = few >> i & 1 && !(few & ((1u << i) - 1)) ? x[i] : one;
                    if (bin(one) != hit) continue;
                    const u64 v = by_weight ? weight(one) : 1;
                    if (v > 0) add_one<by_weight>((int)((hi - key(one)) >> shift), v);
                }
            });
            if (first && cut.ties > 0 && cut.x >= bottom && cut.x <= most && bin(cut.x) == hit)
                add_one<by_weight>((int)((hi - key(cut.x)) >> shift), (u64)cut.ties * (by_weight ? weight(cut.x) : 1));
            const uint32_t at = (uint32_t)find(((int)((hi - lo) >> shift) | 31) + 1, before, target, -1.f);
            const uint32_t key_hi = hi - min(at << shift, hi - lo);            // not below lo: the range shrinks whatever the sums are, and the search ends
            most = of_key(key_hi);
            if (shift == 0) break;
            bottom = of_key(max(lo, key_hi - ((1u << shift) - 1)));
        }
        const u64 one = by_weight ? weight(most) : 1;
        return Cut{most, (int)((target - before + one - 1) / one)};
    }

    // Draws from what remains behind `cut` (greedy: the first of the largest); returns the token.
    __device__ __forceinline__ int draw(const Cut &cut, float u, bool greedy, float &logit)
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        // a warp has consecutive blocks, 32 at a time; an entry sums up 1 << fold of these steps
        const int steps = ((q1 - q0 + kWarps - 1) / kWarps + 31) / 32, own = (w1 - w0 + 31) / 32;
        int fold = 0;
        while (((steps + (1 << fold) - 1) >> fold) > kSteps) ++fold;
        u64 w_warp = 0, w = 0;
        int n_warp = 0, n = 0;
        each_block(w0, w1, 32, [&](const float (&x)[kVec], int j) {
            sums(x, cut, w, n);
            if ((j + 1) % (1 << fold) != 0 && j + 1 < own) return;
            const bool some = __any_sync(0xFFFFFFFFu, w != 0 || n != 0);
            if (some) {
                w = sum_warp(w);
                n = __reduce_add_sync(0xFFFFFFFFu, n);
            }
            if (lane == 0) {
                s.weight[warp][j >> fold] = w;
                s.ties[warp][j >> fold] = n;
            }
            w_warp += w;
            n_warp += n;
            w = 0;
            n = 0;
        });
        const int mine_entries = (own + (1 << fold) - 1) >> fold;
        if (lane == 0) {
            s.warp_weight[warp] = w_warp;
            s.warp_ties[warp] = n_warp;
        }
        __syncthreads();
        // every warp: sums before it in the CTA
        const u64 w_lane = lane < kWarps ? s.warp_weight[lane] : 0;
        const int n_lane = lane < kWarps ? s.warp_ties[lane] : 0;
        const u64 w_scan = scan_warp(w_lane);
        const int n_scan = scan_warp(n_lane);
        if (threadIdx.x == 0) s.token = -1;
        if (warp == 0) {
            const u64 w_sum = __shfl_sync(0xFFFFFFFFu, w_scan, 31);
            const int n_sum = __shfl_sync(0xFFFFFFFFu, n_scan, 31);
            if (lane < (int)ctas) {
                *in_cta(&s.total[rank], lane) = w_sum;
                *in_cta(&s.tied[rank], lane) = n_sum;
            }
        }
        const u64 tie = cut.ties > 0 ? weight(cut.x) : 0;
        cluster_sync_all();
        u64 whole = (u64)cut.ties * tie, w_before = __shfl_sync(0xFFFFFFFFu, w_scan - w_lane, warp);
        int n_before = __shfl_sync(0xFFFFFFFFu, n_scan - n_lane, warp);
#pragma unroll
        for (uint32_t c = 0; c < kMaxCtas; ++c) {
            const u64 v = s.total[c];
            whole += c < ctas ? v : 0;
            w_before += c < rank ? v : 0;
            n_before += c < rank ? s.tied[c] : 0;
        }
        // the first element whose running sum passes `aim`
        const u64 aim = greedy ? 0 : target_of(u, whole);
        auto running = [&](u64 weight_before, int ties_before) { return weight_before + (u64)min(ties_before, cut.ties) * tie; };
        if (running(w_before, n_before) <= aim && running(w_before + w_warp, n_before + n_warp) > aim) {     // one warp of the cluster
            // the entry
            int e = 0;
            if (mine_entries > 1)
                while (true) {
                    const u64 w = e + lane < mine_entries ? s.weight[warp][e + lane] : 0;
                    const int n = e + lane < mine_entries ? s.ties[warp][e + lane] : 0;
                    const u64 ws = scan_warp(w);
                    const int ns = scan_warp(n);
                    const unsigned m = __ballot_sync(0xFFFFFFFFu, running(w_before + ws, n_before + ns) > aim);
                    const int l = m ? __ffs(m) - 1 : 31;
                    w_before += __shfl_sync(0xFFFFFFFFu, m ? ws - w : ws, l);
                    n_before += __shfl_sync(0xFFFFFFFFu, m ? ns - n : ns, l);
                    if (m || e + 32 >= mine_entries) {
                        e = min(e + l, mine_entries - 1);
                        break;
                    }
                    e += 32;
                }
            // its step, lane and element
            for (int j = e << fold; j < own; ++j) {
                float x[kVec];
                u64 w = 0;
                int n = 0;
                const int q = w0 + j * 32 + lane;
#pragma unroll
                for (int i = 0; i < kVec; ++i) x[i] = -INFINITY;
                if (q < w1) block(q, x);
                sums(x, cut, w, n);
                const u64 ws = scan_warp(w);
                const int ns = scan_warp(n);
                const unsigned m = __ballot_sync(0xFFFFFFFFu, running(w_before + ws, n_before + ns) > aim);
                if (m == 0) {
                    w_before += __shfl_sync(0xFFFFFFFFu, ws, 31);
                    n_before += __shfl_sync(0xFFFFFFFFu, ns, 31);
                    continue;
                }
                // element i of that lane's block is looked at by lane i
                const int l = __ffs(m) - 1;
                w_before += __shfl_sync(0xFFFFFFFFu, ws - w, l);
                n_before += __shfl_sync(0xFFFFFFFFu, ns - n, l);
                float mine = -INFINITY;
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float y = __shfl_sync(0xFFFFFFFFu, x[i], l);
                    if (lane == i) mine = y;
                }
                const u64 one = weight(mine), we = scan_warp(mine > cut.x ? one : 0);
                const int ne = scan_warp((int)(mine == cut.x));
                const int i = __ffs(__ballot_sync(0xFFFFFFFFu, running(w_before + we, n_before + ne) > aim)) - 1;
                const int token = (w0 + j * 32 + l) * kVec + i - row.first;
                mine = __shfl_sync(0xFFFFFFFFu, mine, i);
                if (lane < (int)ctas) {
                    *in_cta(&s.token, lane) = token;
                    *in_cta(&s.logit, lane) = mine;
                }
                break;
            }
        }
        if (threadIdx.x == 32 && rank == 0) s.log_whole = ::log((double)whole / kOne);      // meanwhile
        cluster_sync_all();
        logit = s.logit;
        return s.token;
    }
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const SampleArgs a, int cached)
{
    extern __shared__ __align__(16) uint8_t smem[];
    Shared &s = *reinterpret_cast<Shared *>(smem);
    uint4 *cache = reinterpret_cast<uint4 *>(smem + sizeof(Shared));
    const uint32_t rank = cluster_ctarank(), ctas = a.ctas;
    const int b = blockIdx.x / ctas;
    cluster_arrive();                                         // waited for in the first row's maximum()
    if (threadIdx.x < kTable) s.table[threadIdx.x] = __double2ll_rn(exp2(62. - (double)threadIdx.x / kTable));
    pdl_wait();
    pdl_launch_dependents();
    const int n = a.n, L = a.L;
    const int32_t *drafts = a.drafts + (long long)b * n * L;
    const float temperature = a.temperature ? a.temperature[b] : 1.f;
    const bool greedy = !(temperature > 0.f);
    const int top_k = a.top_k ? a.top_k[b] : 0;
    const float top_p = a.top_p ? a.top_p[b] : 1.f;
    const T *logits = static_cast<const T *>(a.logits) + (long long)b * a.chunk_stride;
    // live drafts, one bit each; the same in every thread
    unsigned live = 0;
    for (int r = 0; r < n; ++r) live |= (a.valid[(long long)b * n + r] != 0 ? 1u : 0u) << r;
    int best = __ffs(live) - 1, t = 0;
    // 64 log2(e) / T has to be finite (from 10^-37 down it is not, and weights were no numbers), and the low part of log2(e) / T needs its bits (at
    // 10^36 it is a subnormal number with six, and weights were off by 2^-27)
    if (threadIdx.x == 64) Sampler<T>::set_rate(s, greedy ? 1. : 1.4426950408889634 / (double)fminf(fmaxf(temperature, 1e-36f), 1e33f));
    while (true) {
        const int at = t == 0 ? 0 : 1 + best * L + t - 1;
        Sampler<T> one(s, cache, cached, rank, ctas, logits + (long long)at * a.row_stride, a.V);
        const float u = a.uniform[(long long)b * (L + 1) + t];
        one.clear(0, 0);
        if (threadIdx.x == 0) s.few_count = 0;
        float mine;
        const int valid = one.maximum(mine, t == 0);
        one.scales();
        float logit = 0.f;
        int token = -1;
        const bool cut_k = !greedy && top_k > 0 && top_k < valid;
        if (valid > 0 && !(cut_k && top_k <= kFewKept && one.row.blocks >= 4 * top_k && one.few(top_k, top_p, u, mine, logit, token))) {
            Cut cut{-INFINITY, 0};
            if (greedy) cut = Cut{one.top, 1};
            if (cut_k) cut = one.template select<false>(cut, 0.f, top_k);
            if (!greedy && top_p < 1.f) cut = one.template select<true>(cut, fmaxf(top_p, 0.f), 0);
            token = one.draw(cut, u, greedy, logit);
        }
        if (rank == 0 && threadIdx.x == 0) {
            a.out_tokens[(long long)b * (L + 1) + t] = token;
            if (a.out_logs)
                a.out_logs[(long long)b * (L + 1) + t] =
                    greedy || token < 0 ? 0.f : (float)((logit == one.top ? 0. : ((double)logit - (double)one.top) * (s.rate * 0.6931471805599453)) - s.log_whole);
        }
        ++t;
        unsigned next = 0;
        if (t <= L && token >= 0)
            for (unsigned m = live; m; m &= m - 1) {
                const int r = __ffs(m) - 1;
                if (drafts[r * L + t - 1] == token) next |= 1u << r;
            }
        if (next == 0) break;
        live = next;
        best = __ffs(live) - 1;
    }
    if (rank == 0) {
        if (threadIdx.x == 0) {
            a.out_best[b] = best;
            a.out_len[b] = t;
        }
        for (int i = t + threadIdx.x; i <= L; i += kThreads) {
            a.out_tokens[(long long)b * (L + 1) + i] = -1;
            if (a.out_logs) a.out_logs[(long long)b * (L + 1) + i] = 0.f;
        }
    }
    cluster_sync_all();                                       // a row without logits leaves the others' words unread until here
}

constexpr int kRoom[2] = {112 * 1024, 225 * 1024};            // shared memory of a CTA: two a SM, or one

// Clusters of `ctas` that are resident at once, with kRoom[which].  A cluster lies in one GPC, and some have fewer SMs than others (of 16 CTAs, two a
// SM: 14 clusters, not 18).
template <typename T> cudaError_t resident(int dev, int ctas, int which, int sms, int *clusters)
{
    static std::atomic<int> known[64][kMaxCtas + 1][2];       // by device; + 1
    *clusters = ctas == 1 ? (2 - which) * sms : dev < 64 ? known[dev][ctas][which].load() - 1 : -1;
    if (*clusters >= 0) return cudaSuccess;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kRoom[which];
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaOccupancyMaxActiveClusters(clusters, sample_kernel<T>, &cfg);
    if (e == cudaSuccess && dev < 64) known[dev][ctas][which].store(*clusters + 1);
    return e;
}

template <typename T> cudaError_t launch(SampleArgs a, int sms, cudaStream_t stream)
{
    static std::atomic<bool> ready[64];                       // by device
    int dev = 0, clusters = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev >= 64 || !ready[dev])) {
        e = cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRoom[1]);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e == cudaSuccess && dev < 64) ready[dev] = true;
    }
    if (e != cudaSuccess) return e;
    // CTAs of a cluster: as many as there is room for at two a SM, each with 1024 logits at least.  Without drafts all rows take the same time, and those
    // that wait double the call's (16 rows of 32000, top_k: clusters of 16 23.3 us, of 8 12.5); with drafts sequences
    // end one by one, and a few may wait (16 sequences, 3 x 20 of 100003: 77 us, 88).
    a.ctas = 1;
    while (a.ctas < kMaxCtas && a.B * a.ctas * 2 <= 2 * sms && a.V / (a.ctas * 2) >= 1024) a.ctas *= 2;
    for (; a.n == 0 && a.ctas > 1; a.ctas /= 2) {
        if ((e = resident<T>(dev, a.ctas, 0, sms, &clusters)) != cudaSuccess) return e;
        if (clusters >= a.B) break;
    }
    // a row's piece is kept in shared memory as far as it goes; with one CTA a SM if all clusters find room so
    const int vec = 16 / (int)sizeof(T), blocks = (a.V + 2 * vec - 2) / vec, per = (blocks + a.ctas - 1) / a.ctas;
    int room = (int)((kRoom[0] - sizeof(Shared)) / 16);
    if (per > room) {
        if ((e = resident<T>(dev, a.ctas, 1, sms, &clusters)) != cudaSuccess) return e;
        if (clusters >= a.B) room = (int)((kRoom[1] - sizeof(Shared)) / 16);
    }
    const int cached = per < room ? per : room;
    const size_t smem = sizeof(Shared) + 16 * (size_t)cached;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = a.ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.gridDim = dim3(a.B * a.ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, sample_kernel<T>, a, cached);
}

}  // namespace

cudaError_t launch_sample(const SampleArgs &a, int dtype, int sms, cudaStream_t stream)
{
    return dtype == kF16 ? launch<__half>(a, sms, stream) : dtype == kBF16 ? launch<__nv_bfloat16>(a, sms, stream) : launch<float>(a, sms, stream);
}

}  // namespace dresd
