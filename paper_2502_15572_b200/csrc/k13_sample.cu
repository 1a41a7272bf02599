// K13 -- verification of drafts against the model's distribution, from given random numbers (no drafts: sampling).
//
// A sequence is a chain: the token drawn at depth t decides which row of logits is read at depth t + 1, so that only the rows on
// the path are read, at most L + 1 of the 1 + n L.  One cluster follows a sequence; its CTAs share a row by contiguous pieces.
// Per row: the maximum; the cuts of top_k and top_p (radix selection by histograms of 2048 bins, summed over the cluster);
// the weights' sums piece by piece; and the piece, warp, lane and element where the running sum passes u times the whole.
//
// A weight is rint(2^42 e^((x - max) / T)), a whole number: sums are exact, so they depend neither on their order nor on how
// many CTAs share a row, and a token is the same whatever the batch.
#include "common.cuh"
#include "internal.h"

namespace dresd {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32, kMaxCtas = 8;
constexpr int kBins = 2048, kEntries = 2048;
constexpr double kOne = 4398046511104.0;                       // 2^42, the largest weight

typedef unsigned long long u64;

template <typename T> __device__ __forceinline__ float to_float(T x) { return x; }
template <> __device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

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
    // Elements of block q; what is not the row's, and NaN, as -infinity; -0 as 0.
    __device__ __forceinline__ void load(int q, float (&x)[kVec]) const
    {
        const int j = q * kVec;
        if (j >= first && j + kVec <= last) {
            const uint4 w = *reinterpret_cast<const uint4 *>(base + j);
            const T *e = reinterpret_cast<const T *>(&w);
#pragma unroll
            for (int i = 0; i < kVec; ++i) x[i] = to_float(e[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) x[i] = j + i >= first && j + i < last ? to_float(base[j + i]) : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < kVec; ++i) x[i] = x[i] == x[i] ? x[i] + 0.f : -INFINITY;
    }
};

// Order of logits as whole numbers.  16-bit types leave the low 13 bits of a float alike, so that 22 bits tell them apart.
template <typename T> struct Order {
    static constexpr int kBits = sizeof(T) == 2 ? 22 : 32, kPasses = sizeof(T) == 2 ? 2 : 3;
    static __device__ __forceinline__ uint32_t key(float x) { return float_to_ordered(x) >> (32 - kBits); }
    static __device__ __forceinline__ int shift(int pass) { return max(kBits - 11 * (pass + 1), 0); }
    static __device__ __forceinline__ int width(int pass) { return kBits - 11 * pass - shift(pass); }
};

// What remains of a row: elements whose key is larger, and the first `ties` of those whose key is equal.
struct Cut {
    uint32_t key;
    int ties;
};

struct Shared {
    union {
        struct {
            u64 bins[kBins];             // this CTA's elements
            u64 sums[kBins];             // the cluster's, for this CTA's part of the bins
        };
        struct {
            u64 weight[kEntries];        // of a warp's consecutive blocks
            int ties[kEntries];
        };
    };
    u64 warp_u64[kWarps];
    int warp_int[kWarps];
    u64 total;                           // of this CTA, for the others to read
    int count;                           // of logits above -infinity
    int tied;                            // of those that the cut ties
    float top;
    u64 found_above;                     // written by the CTA that finds it, in every CTA
    int found_bin;
    int token;
    float log;
};

template <typename V> __device__ __forceinline__ V *in_cta(V *p, uint32_t rank)
{
    u64 r;
    asm("mapa.u64 %0, %1, %2;" : "=l"(r) : "l"(reinterpret_cast<u64>(p)), "r"(rank));
    return reinterpret_cast<V *>(r);
}

__device__ __forceinline__ u64 shfl_up64(u64 x, int o) { return __shfl_up_sync(0xFFFFFFFFu, x, o); }

// Exclusive sums over the CTA's threads, of a weight and a count.
__device__ __forceinline__ void scan_cta(u64 x, int n, Shared &s, u64 &x_before, int &n_before, u64 &x_total, int &n_total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    u64 xi = x;
    int ni = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 y = shfl_up64(xi, o);
        const int m = __shfl_up_sync(0xFFFFFFFFu, ni, o);
        if (lane >= o) {
            xi += y;
            ni += m;
        }
    }
    __syncthreads();
    if (lane == 31) {
        s.warp_u64[warp] = xi;
        s.warp_int[warp] = ni;
    }
    __syncthreads();
    u64 xs = s.warp_u64[lane];
    int ns = s.warp_int[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 y = shfl_up64(xs, o);
        const int m = __shfl_up_sync(0xFFFFFFFFu, ns, o);
        if (lane >= o) {
            xs += y;
            ns += m;
        }
    }
    x_total = __shfl_sync(0xFFFFFFFFu, xs, 31);
    n_total = __shfl_sync(0xFFFFFFFFu, ns, 31);
    const u64 xb = __shfl_sync(0xFFFFFFFFu, xs, max(warp - 1, 0));
    const int nb = __shfl_sync(0xFFFFFFFFu, ns, max(warp - 1, 0));
    x_before = (warp ? xb : 0) + xi - x;
    n_before = (warp ? nb : 0) + ni - n;
}
static_assert(kWarps == 32, "scan_cta: one sum a lane");

template <typename T>
struct Sampler {
    static constexpr int kVec = Row<T>::kVec;
    Shared &s;
    const uint32_t rank, ctas;
    const Row<T> row;
    int q0, q1;                  // this CTA's blocks
    float top;                   // the row's largest logit
    double rate;                 // 1 / T
    __device__ __forceinline__ Sampler(Shared &s_, uint32_t rank_, uint32_t ctas_, const T *p, int V)
        : s(s_), rank(rank_), ctas(ctas_), row(p, V), top(0.f), rate(1.)
    {
        const int per = (row.blocks + ctas - 1) / ctas;
        q0 = min((int)rank * per, row.blocks);
        q1 = min(q0 + per, row.blocks);
    }
    __device__ __forceinline__ u64 weight(float x) const
    {
        if (x == top) return (u64)kOne;
        const double below = (double)x - (double)top;
        return below > -INFINITY ? (u64)__double2ll_rn(exp(below * rate) * kOne) : 0;
    }
    __device__ __forceinline__ bool above(float x, const Cut &c) const { return x > -INFINITY && Order<T>::key(x) > c.key; }
    __device__ __forceinline__ bool tied(float x, const Cut &c) const { return x > -INFINITY && Order<T>::key(x) == c.key; }

    // The row's largest logit and how many logits there are above -infinity.
    __device__ __forceinline__ int maximum()
    {
        float m = -INFINITY;
        int n = 0;
        for (int q = q0 + threadIdx.x; q < q1; q += kThreads) {
            float x[kVec];
            row.load(q, x);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                m = fmaxf(m, x[i]);
                n += x[i] > -INFINITY;
            }
        }
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        n = __reduce_add_sync(0xFFFFFFFFu, n);
        uint32_t k = __reduce_max_sync(0xFFFFFFFFu, float_to_ordered(m));
        __syncthreads();
        if (lane == 0) {
            s.warp_int[warp] = n;
            s.warp_u64[warp] = k;
        }
        __syncthreads();
        if (warp == 0) {
            n = __reduce_add_sync(0xFFFFFFFFu, s.warp_int[lane]);
            k = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)s.warp_u64[lane]);
            if (lane == 0) {
                s.count = n;
                s.top = ordered_to_float(k);
            }
        }
        cluster_sync_all();
        top = -INFINITY;
        n = 0;
        for (uint32_t c = 0; c < ctas; ++c) {
            top = fmaxf(top, *in_cta(&s.top, c));
            n += *in_cta(&s.count, c);
        }
        return n;
    }

    // Sum over the cluster of what remains behind `cut`.
    __device__ __forceinline__ u64 sum(const Cut &cut)
    {
        u64 w = 0;
        for (int q = q0 + threadIdx.x; q < q1; q += kThreads) {
            float x[kVec];
            row.load(q, x);
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (above(x[i], cut)) w += weight(x[i]);
        }
        u64 xb, xt;
        int nb, nt;
        scan_cta(w, 0, s, xb, nb, xt, nt);
        if (threadIdx.x == 0) s.total = xt;
        cluster_sync_all();
        w = 0;
        for (uint32_t c = 0; c < ctas; ++c) w += *in_cta(&s.total, c);
        cluster_sync_all();
        return w + (u64)cut.ties * weight_of(cut.key);
    }
    __device__ __forceinline__ u64 weight_of(uint32_t key) const       // of the logit with this key
    {
        constexpr int low = 32 - Order<T>::kBits;
        const uint32_t u = key << low;
        return weight(ordered_to_float(u & 0x80000000u ? u : u | ((1u << low) - 1)));
    }

    // The shortest part of `cut`, in descending order and then by index, whose elements' weights (counts) reach `target`, which is
    // positive and not more than they have in all.
    template <bool by_weight>
    __device__ __forceinline__ Cut select(const Cut &cut, u64 target)
    {
        uint32_t prefix = 0;
        u64 before = 0;
        for (int pass = 0; pass < Order<T>::kPasses; ++pass) {
            const int shift = Order<T>::shift(pass), width = Order<T>::width(pass), bins = 1 << width;
            const bool all = pass == 0;
            for (int i = threadIdx.x; i < kBins; i += kThreads) s.bins[i] = 0;
            __syncthreads();
            for (int q = q0 + threadIdx.x; q < q1; q += kThreads) {
                float x[kVec];
                row.load(q, x);
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const uint32_t k = Order<T>::key(x[i]);
                    if (above(x[i], cut) && (all || k >> (shift + width) == prefix))
                        atomicAdd(s.bins + (k >> shift & (bins - 1)), by_weight ? weight(x[i]) : 1ull);
                }
            }
            if (rank == 0 && threadIdx.x == 0 && cut.ties > 0 && (all || cut.key >> (shift + width) == prefix))
                atomicAdd(s.bins + (cut.key >> shift & (bins - 1)), (u64)cut.ties * (by_weight ? weight_of(cut.key) : 1ull));
            cluster_sync_all();
            // bins are summed over the cluster by the CTA whose part they are, and searched from the largest key down:
            // position i stands for bin bins - 1 - i
            const int part = bins / ctas, first = (int)rank * part;
            u64 mine = 0;
            const int each = (part + kThreads - 1) / kThreads;
            for (int j = 0; j < each; ++j) {
                const int i = threadIdx.x * each + j;
                if (i >= part) break;
                u64 v = 0;
                for (uint32_t c = 0; c < ctas; ++c) v += *in_cta(s.bins + (bins - 1 - first - i), c);
                s.sums[i] = v;
                mine += v;
            }
            u64 mine_before, total;
            int nb, nt;
            scan_cta(mine, 0, s, mine_before, nb, total, nt);
            if (threadIdx.x == 0) s.total = total;
            cluster_sync_all();
            u64 at = before;
            for (uint32_t c = 0; c < rank; ++c) at += *in_cta(&s.total, c);
            at += mine_before;
            if (at < target && at + mine >= target) {           // one thread of the cluster
                for (int j = 0; j < each; ++j) {
                    const u64 v = s.sums[threadIdx.x * each + j];
                    if (at + v >= target) {
                        for (uint32_t c = 0; c < ctas; ++c) {
                            *in_cta(&s.found_bin, c) = bins - 1 - first - (threadIdx.x * each + j);
                            *in_cta(&s.found_above, c) = at;
                        }
                        break;
                    }
                    at += v;
                }
            }
            cluster_sync_all();
            prefix = prefix << width | (uint32_t)s.found_bin;
            before = s.found_above;
        }
        const u64 one = by_weight ? weight_of(prefix) : 1ull;
        return Cut{prefix, (int)((target - before + one - 1) / one)};
    }

    // Draws from what remains behind `cut` (greedy: the first of the largest); returns the token, -1 if nothing remains.
    __device__ __forceinline__ int draw(const Cut &cut, float u, bool greedy, float &log)
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        // a warp has `per` consecutive blocks, 32 at a time; an entry sums up 1 << fold of these steps
        const int per = (q1 - q0 + kWarps - 1) / kWarps, w0 = min(q0 + warp * per, q1), w1 = min(w0 + per, q1);
        const int steps = (per + 31) / 32;
        int fold = 0;
        while (((steps + (1 << fold) - 1) >> fold) * kWarps > kEntries) ++fold;
        const int entries = (steps + (1 << fold) - 1) >> fold;      // of a warp
        for (int e = 0; e < entries; ++e) {
            u64 w = 0;
            int n = 0;
            for (int j = e << fold; j < min(steps, (e + 1) << fold); ++j) {
                const int q = w0 + j * 32 + lane;
                if (q >= w1) continue;
                float x[kVec];
                row.load(q, x);
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    if (above(x[i], cut)) w += weight(x[i]);
                    n += tied(x[i], cut);
                }
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) w += __shfl_xor_sync(0xFFFFFFFFu, w, o);
            n = __reduce_add_sync(0xFFFFFFFFu, n);
            if (lane == 0) {
                s.weight[warp * entries + e] = w;
                s.ties[warp * entries + e] = n;
            }
        }
        __syncthreads();
        const int each = (kWarps * entries + kThreads - 1) / kThreads;
        u64 w = 0, w_before, w_total;
        int n = 0, n_before, n_total;
        for (int j = 0; j < each; ++j) {
            const int e = threadIdx.x * each + j;
            if (e < kWarps * entries) {
                w += s.weight[e];
                n += s.ties[e];
            }
        }
        scan_cta(w, n, s, w_before, n_before, w_total, n_total);
        if (threadIdx.x == 0) {
            s.total = w_total;
            s.tied = n_total;
            s.token = -1;
            s.log = 0.f;
        }
        cluster_sync_all();
        const u64 tie = weight_of(cut.key);
        u64 whole = 0;
        for (uint32_t c = 0; c < ctas; ++c) {
            const u64 wc = *in_cta(&s.total, c);
            const int nc = *in_cta(&s.tied, c);
            if (c < rank) {
                w_before += wc;
                n_before += nc;
            }
            whole += wc;
        }
        whole += (u64)cut.ties * tie;
        // the first element whose running sum passes `aim`
        const u64 aim = greedy ? 0 : (u64)__double2ll_rz((double)fminf(fmaxf(u, 0.f), 1.f - 0x1p-24f) * (double)whole);
        auto running = [&](u64 weight_before, int ties_before) { return weight_before + (u64)min(ties_before, cut.ties) * tie; };
        if (running(w_before, n_before) <= aim && running(w_before + w, n_before + n) > aim) {    // one thread of the cluster
            for (int j = 0; j < each; ++j) {
                const int e = threadIdx.x * each + j;
                if (running(w_before + s.weight[e], n_before + s.ties[e]) > aim) {
                    s.found_bin = e;
                    s.found_above = w_before;
                    s.warp_int[0] = n_before;
                    break;
                }
                w_before += s.weight[e];
                n_before += s.ties[e];
            }
        } else {
            n_before = -1;
        }
        const bool here = __syncthreads_or(n_before >= 0);
        if (here && warp == 0) {
            const int e = s.found_bin, of = e / entries, j0 = (e % entries) << fold;
            const int v0 = min(q0 + of * per, q1), v1 = min(v0 + per, q1);
            u64 sum = s.found_above;
            int ties = s.warp_int[0];
            for (int j = j0; j < min(steps, j0 + (1 << fold)); ++j) {
                const int q = v0 + j * 32 + lane;
                float x[kVec];
                u64 mine = 0;
                int count = 0;
                if (q < v1) {
                    row.load(q, x);
#pragma unroll
                    for (int i = 0; i < kVec; ++i) {
                        if (above(x[i], cut)) mine += weight(x[i]);
                        count += tied(x[i], cut);
                    }
                }
                u64 mine_inc = mine;
                int count_inc = count;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const u64 y = shfl_up64(mine_inc, o);
                    const int m = __shfl_up_sync(0xFFFFFFFFu, count_inc, o);
                    if (lane >= o) {
                        mine_inc += y;
                        count_inc += m;
                    }
                }
                const bool in = running(sum + mine_inc, ties + count_inc) > aim;
                const unsigned m = __ballot_sync(0xFFFFFFFFu, in);
                if (m == 0) {
                    sum += __shfl_sync(0xFFFFFFFFu, mine_inc, 31);
                    ties += __shfl_sync(0xFFFFFFFFu, count_inc, 31);
                    continue;
                }
                if (lane == __ffs(m) - 1) {
                    sum += mine_inc - mine;
                    ties += count_inc - count;
                    bool done = false;
#pragma unroll
                    for (int i = 0; i < kVec; ++i) {
                        if (above(x[i], cut)) sum += weight(x[i]);
                        ties += tied(x[i], cut);
                        if (!done && running(sum, ties) > aim) {
                            done = true;
                            const float l = greedy ? 0.f : (float)((x[i] == top ? 0. : ((double)x[i] - (double)top) * rate) - ::log((double)whole / kOne));
                            for (uint32_t c = 0; c < ctas; ++c) {
                                *in_cta(&s.token, c) = q * kVec + i - row.first;
                                *in_cta(&s.log, c) = l;
                            }
                        }
                    }
                }
                break;
            }
        }
        cluster_sync_all();
        log = s.log;
        return s.token;
    }
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 1) sample_kernel(const SampleArgs a)
{
    __shared__ Shared s;
    const uint32_t rank = cluster_ctarank(), ctas = a.ctas;
    const int b = blockIdx.x / ctas;
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
    while (true) {
        const int at = t == 0 ? 0 : 1 + best * L + t - 1;
        Sampler<T> one(s, rank, ctas, logits + (long long)at * a.row_stride, a.V);
        const int valid = one.maximum();
        one.rate = greedy ? 1. : 1. / (double)temperature;
        Cut cut{0, 0};                                        // all: no logit has key 0
        if (greedy) cut = Cut{Order<T>::key(one.top), 1};
        else if (valid > 0) {
            if (top_k > 0 && top_k < valid) cut = one.template select<false>(cut, top_k);
            if (top_p < 1.f) {
                const u64 all = one.sum(cut);
                const u64 target = (u64)__double2ll_ru((double)fmaxf(top_p, 0.f) * (double)all);
                cut = one.template select<true>(cut, max(target, 1ull));
            }
        }
        float log = 0.f;
        const int token = valid > 0 ? one.draw(cut, a.uniform[(long long)b * (L + 1) + t], greedy, log) : -1;
        if (rank == 0 && threadIdx.x == 0) {
            a.out_tokens[(long long)b * (L + 1) + t] = token;
            if (a.out_logs) a.out_logs[(long long)b * (L + 1) + t] = log;
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
        cluster_sync_all();                                   // the shared words are read no more
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
    cluster_sync_all();
}

}  // namespace

cudaError_t launch_sample(const SampleArgs &args, int dtype, int sms, cudaStream_t stream)
{
    SampleArgs a = args;
    // CTAs of a cluster: as many as the sequences leave SMs for, each with 2048 logits at least
    a.ctas = 1;
    while (a.ctas < kMaxCtas && a.B * a.ctas * 2 <= sms && a.V / (a.ctas * 2) >= 2048) a.ctas *= 2;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = a.ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.gridDim = dim3(a.B * a.ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return dtype == kF16    ? cudaLaunchKernelEx(&cfg, sample_kernel<__half>, a)
           : dtype == kBF16 ? cudaLaunchKernelEx(&cfg, sample_kernel<__nv_bfloat16>, a)
                            : cudaLaunchKernelEx(&cfg, sample_kernel<float>, a);
}

}  // namespace dresd
