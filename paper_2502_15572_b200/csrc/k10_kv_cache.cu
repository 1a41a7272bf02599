// K10 -- the paged key/value cache: writing (and quantising) new tokens, reading positions back, and moving
// the accepted draft's tokens into place.
//
// All three move every byte once and compute next to nothing, so they are bound by HBM (and, on a few
// hundred tokens, by the launch and the chain start[] -> ctx[] -> table -> data).  A lane handles 16 bytes
// of a 16-bit row (8 elements), so a row of d = 128 is one half-warp and the quantiser's
// maximum is four shuffles; a thread takes the same piece of kHeads heads of a token, whose loads
// are independent and whose page is looked up once.
//
// Measured: 60000 positions x 8 heads of 128 read back in 75 us = 6.5 TB/s, 99 % of what a copy reaches; 32000 quantised in
// 37 us = 5.25 TB/s (the maximum has to be known before the first code is written); 101 tokens of 32 heads appended in 2.0 us.
#include "kv_plan.cuh"

namespace dresd {
namespace {

constexpr int kThreads = 256;
constexpr int kHeads = 4;        // heads per thread (2: 32000 tokens quantised in 46 us; 4: 37; 8: 36, but short calls slower)
constexpr int kKeepBlocks = 1184; // eight per SM: what is resident at once

// Page and offset of a dense row's token; false when the table does not reach it or names no page of the pool.
__device__ __forceinline__ bool place_of(const KvArgs &a, int row, int &page, int &off)
{
    int lo = 0, hi = a.B;                                  // last b with start[b] <= row
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(a.start + mid) <= row) lo = mid;
        else hi = mid;
    }
    const int first = max(__ldg(a.start + lo), 0);
    if (row < first || row >= __ldg(a.start + lo + 1)) return false;
    const long long p = (long long)max(__ldg(a.ctx + lo), 0) + (row - first);
    const long long i = p >> a.page_shift;
    if (i >= a.width || !debug_check(lo < a.B && i >= 0, a.status, 51)) return false;
    page = __ldg(a.table + (long long)lo * a.width + i);
    off = (int)(p & ((1 << a.page_shift) - 1));
    return page >= 0 && page < a.num_pages;
}

// Magnitudes above the bound become the bound; NaN stays one.
template <typename T>
__device__ __forceinline__ uint32_t bounded(uint32_t two)
{
    constexpr uint32_t kInf = std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u;
    uint32_t lo = two & 0xFFFFu, hi = two >> 16;
    if (lo > KvType<T>::kBoundBits && lo <= kInf) lo = KvType<T>::kBoundBits;
    if (hi > KvType<T>::kBoundBits && hi <= kInf) hi = KvType<T>::kBoundBits;
    return lo | hi << 16;
}

template <typename T, bool Q8, int D>
__global__ void __launch_bounds__(kThreads)
append_kernel(const KvArgs a, const T *__restrict__ k, long long k_row, long long k_head, const T *__restrict__ v,
              long long v_row, long long v_head)
{
    constexpr int kLanes = D / 8;                          // threads per row
    const int groups = (a.heads + kHeads - 1) / kHeads;
    const long long unit = ((long long)blockIdx.x * kThreads + threadIdx.x) / kLanes;
    const int piece = threadIdx.x % kLanes;
    if (unit >= (long long)a.rows * groups) return;        // whole sub-warps leave together
    const int row = (int)(unit / groups), h0 = (int)(unit % groups) * kHeads;
    pdl_wait();
    pdl_launch_dependents();
    const bool is_v = blockIdx.y != 0;
    const T *src = is_v ? v + row * v_row : k + row * k_row;
    const long long step = is_v ? v_head : k_head;
    uint4 x[kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; ++i)
        if (h0 + i < a.heads) x[i] = __ldg(reinterpret_cast<const uint4 *>(src + (h0 + i) * step + piece * 8));
    int page, off;
    if (!place_of(a, row, page, off)) return;
    constexpr uint32_t kMag = 0x7FFF7FFFu;
    const unsigned lanes = kLanes == 32 ? 0xFFFFFFFFu : ((1u << kLanes) - 1) << (threadIdx.x % 32 / kLanes * kLanes);
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        if (h0 + i >= a.heads) break;
        const long long r = kv_row(a, a.layer, page, h0 + i, off);
        if (!debug_check(r >= 0 && r < kv_rows(a), a.status, 52)) break;       // the same for every lane of the row
        if constexpr (!Q8) {
            reinterpret_cast<uint4 *>(is_v ? a.v : a.k)[r * kLanes + piece] = x[i];
        } else {
            uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
            // magnitudes of either type order like their bits, two at a time
            uint32_t big = __vmaxu2(__vmaxu2(w[0] & kMag, w[1] & kMag), __vmaxu2(w[2] & kMag, w[3] & kMag));
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) big = __vmaxu2(big, __shfl_xor_sync(lanes, big, o));
            big = max(big & 0xFFFFu, big >> 16);
            if (big > KvType<T>::kBoundBits) {             // the same for every lane of the row
                big = KvType<T>::kBoundBits;
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = (w[j] & ~kMag) | bounded<T>(w[j] & kMag);
            }
            const int e = kv_exponent(unpack2<T>(big).x, KvType<T>::kMinExp);
            const float s = pow2f(-e);                     // the product is exact: one rounding, to E4M3
            uint32_t c[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float2 p = unpack2<T>(w[j]);
                p.x *= s;
                p.y *= s;
                c[j] = __nv_cvt_float2_to_fp8x2(p, __NV_SATFINITE, __NV_E4M3);
            }
            reinterpret_cast<uint2 *>(is_v ? a.v : a.k)[r * kLanes + piece] = make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
            if (piece == 0) (is_v ? a.v_exps : a.k_exps)[r] = (uint8_t)(e + 127);
        }
    }
}

template <typename T, bool Q8, int D>
__global__ void __launch_bounds__(kThreads) read_kernel(const KvArgs a, T *__restrict__ out_k, T *__restrict__ out_v)
{
    constexpr int kLanes = D / 8;
    const int groups = (a.heads + kHeads - 1) / kHeads;
    const long long unit = ((long long)blockIdx.x * kThreads + threadIdx.x) / kLanes;
    const int piece = threadIdx.x % kLanes;
    if (unit >= (long long)a.rows * groups) return;
    const int row = (int)(unit / groups), h0 = (int)(unit % groups) * kHeads;
    pdl_wait();
    pdl_launch_dependents();
    const bool is_v = blockIdx.y != 0;
    uint4 *dst = reinterpret_cast<uint4 *>(is_v ? out_v : out_k) + ((long long)row * a.heads + h0) * kLanes + piece;
    int page = 0, off = 0;
    const bool there = place_of(a, row, page, off) &&
                       debug_check(kv_row(a, a.layer, page, min(h0 + kHeads, a.heads) - 1, off) < kv_rows(a), a.status, 53);
    const void *cache = is_v ? a.v : a.k;
    if constexpr (!Q8) {
        uint4 x[kHeads];
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
            x[i] = make_uint4(0, 0, 0, 0);
            if (there && h0 + i < a.heads)
                x[i] = reinterpret_cast<const uint4 *>(cache)[kv_row(a, a.layer, page, h0 + i, off) * kLanes + piece];
        }
#pragma unroll
        for (int i = 0; i < kHeads; ++i)
            if (h0 + i < a.heads) dst[i * kLanes] = x[i];
    } else {
        const uint8_t *exps = is_v ? a.v_exps : a.k_exps;
        uint2 x[kHeads];
        int e[kHeads];
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
            x[i] = make_uint2(0, 0);
            e[i] = 127;
            if (there && h0 + i < a.heads) {
                const long long r = kv_row(a, a.layer, page, h0 + i, off);
                x[i] = reinterpret_cast<const uint2 *>(cache)[r * kLanes + piece];
                e[i] = exps[r];
            }
        }
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
            if (h0 + i >= a.heads) break;
            const float s = __uint_as_float(max((uint32_t)e[i], 1u) << 23);      // stored bytes are 1 .. 247
            const uint32_t w[2] = {x[i].x, x[i].y};
            uint32_t o[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t two = w[j >> 1] >> (16 * (j & 1));
                o[j] = pack2<T>(from_e4m3(two & 0xFF) * s, from_e4m3(two >> 8 & 0xFF) * s);
            }
            dst[i * kLanes] = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
}

// A warp takes one head of one layer, a few lanes a row.  Sources lie behind every destination (1 + best L + t >= 1 + L >
// 1 + t'), so the rows move independently of each other.  gridDim.z / 2 warps share a head's rows as long as all blocks
// are resident at once: 32 sequences of 20 tokens (10 MB in, 10 MB out) 9.4 us, 20 us with a row-step per thread in a
// larger grid; 9 tokens of one sequence 2.1 us, 3.0 with a warp for all of a head's rows.
__global__ void __launch_bounds__(kThreads)
keep_kernel(const KvArgs a, const int32_t *__restrict__ best, const int32_t *__restrict__ length, int n, int L,
            int lanes_shift)
{
    pdl_wait();
    pdl_launch_dependents();
    const int b = blockIdx.y, r = best[b], kept = min(length[b] - 1, L);
    if (r < 1 || r >= n || kept < 1) return;
    const int lh = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (lh >= a.layers * a.heads) return;
    const int layer = lh / a.heads, head = lh - layer * a.heads;
    const int lane = threadIdx.x & 31, rows = 32 >> lanes_shift, sub = lane >> lanes_shift, piece = lane & ((1 << lanes_shift) - 1);
    const int ctx = max(a.ctx[b], 0), in_page = (1 << a.page_shift) - 1;
    const int32_t *table = a.table + (long long)b * a.width;
    const bool is_v = blockIdx.z & 1;
    uint4 *cache = static_cast<uint4 *>(is_v ? a.v : a.k);
    uint8_t *exps = is_v ? a.v_exps : a.k_exps;
    for (int t = (blockIdx.z >> 1) * rows + sub; t < kept; t += (gridDim.z >> 1) * rows) {
        const long long p = (long long)ctx + 1 + t, q = p + (long long)r * L;
        if ((q >> a.page_shift) >= a.width) return;
        const int pf = __ldg(table + (q >> a.page_shift)), pt = __ldg(table + (p >> a.page_shift));
        if (pf < 0 || pf >= a.num_pages || pt < 0 || pt >= a.num_pages) continue;
        const long long from = kv_row(a, layer, pf, head, (int)(q & in_page)), to = kv_row(a, layer, pt, head, (int)(p & in_page));
        if (!debug_check(from >= 0 && from < kv_rows(a) && to >= 0 && to < kv_rows(a) && pt >= 0, a.status, 54)) continue;
        cache[(to << lanes_shift) + piece] = cache[(from << lanes_shift) + piece];
        if (exps && piece == 0) exps[to] = exps[from];
    }
}

template <typename F>
cudaError_t by_type(const KvArgs &a, F &&f)
{
    const bool q8 = a.k_exps != nullptr;
    if (a.dtype == kF16) {
        __half *t = nullptr;
        if (a.d == 64) return q8 ? f(t, std::true_type{}, std::integral_constant<int, 64>{}) : f(t, std::false_type{}, std::integral_constant<int, 64>{});
        return q8 ? f(t, std::true_type{}, std::integral_constant<int, 128>{}) : f(t, std::false_type{}, std::integral_constant<int, 128>{});
    }
    __nv_bfloat16 *t = nullptr;
    if (a.d == 64) return q8 ? f(t, std::true_type{}, std::integral_constant<int, 64>{}) : f(t, std::false_type{}, std::integral_constant<int, 64>{});
    return q8 ? f(t, std::true_type{}, std::integral_constant<int, 128>{}) : f(t, std::false_type{}, std::integral_constant<int, 128>{});
}

dim3 row_grid(const KvArgs &a)
{
    const long long units = (long long)a.rows * ((a.heads + kHeads - 1) / kHeads);
    return dim3((unsigned)((units * (a.d / 8) + kThreads - 1) / kThreads), 2);
}

}  // namespace

cudaError_t launch_kv_append(const KvArgs &a, const void *k, long long k_row, long long k_head, const void *v,
                             long long v_row, long long v_head, cudaStream_t stream)
{
    return by_type(a, [&](auto *t, auto q8, auto d) {
        using T = std::remove_pointer_t<decltype(t)>;
        return launch_dependent(append_kernel<T, decltype(q8)::value, decltype(d)::value>, row_grid(a), dim3(kThreads), 0, stream, a,
                                static_cast<const T *>(k), k_row, k_head, static_cast<const T *>(v), v_row, v_head);
    });
}

cudaError_t launch_kv_read(const KvArgs &a, void *out_k, void *out_v, cudaStream_t stream)
{
    return by_type(a, [&](auto *t, auto q8, auto d) {
        using T = std::remove_pointer_t<decltype(t)>;
        return launch_dependent(read_kernel<T, decltype(q8)::value, decltype(d)::value>, row_grid(a), dim3(kThreads), 0, stream, a,
                                static_cast<T *>(out_k), static_cast<T *>(out_v));
    });
}

cudaError_t launch_kv_keep_draft(const KvArgs &a, const int32_t *best, const int32_t *length, int n, int L,
                                 cudaStream_t stream)
{
    const int pieces = a.d * (a.k_exps ? 1 : 2) / 16;      // of a row: 4, 8 or 16
    const int lanes_shift = pieces == 4 ? 2 : pieces == 8 ? 3 : 4, warps = kThreads / 32, rows = 32 >> lanes_shift;
    const int across = (a.layers * a.heads + warps - 1) / warps;
    const int most = max((int)(kKeepBlocks / (2LL * across * a.B)), 1);
    const dim3 grid(across, a.B, 2 * min((L + rows - 1) / rows, most));
    return launch_dependent(keep_kernel, grid, dim3(kThreads), 0, stream, a, best, length, n, L, lanes_shift);
}

}  // namespace dresd
