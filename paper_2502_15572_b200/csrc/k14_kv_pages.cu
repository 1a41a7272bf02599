// K14 -- pages of the key/value cache: fork (rows become copies of other rows and share their pages), reserve (the places of the
// next chunk become the row's own: absent pages are taken, shared ones replaced and copied), release, compact.
//
// The only state is refs[page] = rows that hold the page; a page is free when that is not positive.  Free pages are taken in
// ascending order and wishes served in the order (row, place), so results do not depend on timing.  Planning is a chain of
// a few dependent loads and cluster barriers (latency); moving pages is a copy (HBM).  Measured (device): compacting 176 MB (read and
// written) 38 us, 1191 MB 211 us (5.65 TB/s, 86 % of the copy rate; 4 us are the plan); forking 24 prompts into 72 rows, reserving 61 places
// each (304 MB) and releasing 62 us, one prompt into 8 (34 MB) 19 us: five launches and what each waits for.
#include "kv_plan.cuh"

namespace dresd {
namespace {

constexpr int kRowThreads = 256;
constexpr int kMaxPlanCtas = 8, kMaxPlanThreads = 1024;      // of the planning cluster: see plan_size()
constexpr int kMoveThreads = 256, kMoveBytes = kMoveThreads * 4 * 16;   // of a piece: four 16-byte loads a thread

__device__ __forceinline__ int places_for(long long tokens, int page_shift, int width)
{
    return (int)min((max(tokens, 0LL) + (1LL << page_shift) - 1) >> page_shift, (long long)width);
}
__device__ __forceinline__ bool is_page(const KvArgs &a, int e) { return e >= 0 && e < a.num_pages; }

// One CTA a row.  Rows that are read have no parent of their own, so nobody writes them.
__global__ void __launch_bounds__(kRowThreads)
fork_kernel(const KvArgs a, int32_t *__restrict__ refs, int32_t *table, int32_t *ctx, const int32_t *__restrict__ parent)
{
    pdl_wait();
    pdl_launch_dependents();
    const int b = blockIdx.x, p = parent[b];
    if (p < 0 || p >= a.B || parent[p] >= 0) return;
    const int tokens = ctx[p], held = places_for(tokens, a.page_shift, a.width);
    const int32_t *from = table + (long long)p * a.width;
    int32_t *to = table + (long long)b * a.width;
    for (int i = threadIdx.x; i < a.width; i += kRowThreads) {
        const int e = i < held ? from[i] : -1;
        to[i] = e;
        if (is_page(a, e)) atomicAdd(refs + e, 1);
    }
    if (threadIdx.x == 0) ctx[b] = tokens;
}

__global__ void __launch_bounds__(kRowThreads)
release_kernel(const KvArgs a, int32_t *__restrict__ refs, int32_t *__restrict__ table, const int32_t *__restrict__ keep)
{
    pdl_wait();
    pdl_launch_dependents();
    int32_t *row = table + (long long)blockIdx.x * a.width;
    for (int i = places_for(keep[blockIdx.x], a.page_shift, a.width) + threadIdx.x; i < a.width; i += kRowThreads) {
        const int e = row[i];
        if (!is_page(a, e)) continue;
        row[i] = -1;
        if (atomicSub(refs + e, 1) <= 0) atomicAdd(refs + e, 1);          // contradictory counts stop at zero
    }
}

// ---- planning: one cluster -------------------------------------------------------------------------------------
__device__ __forceinline__ int load_cluster(const int *p, uint32_t rank)
{
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(mapa_rank(smem_u32(p), rank)) : "memory");
    return v;
}
// Exclusive sum over the CTA's threads; `total` of all.  sums: 32 words.
__device__ __forceinline__ int scan_cta(int x, int *sums, int &total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int inc = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xFFFFFFFFu, inc, o);
        if (lane >= o) inc += y;
    }
    __syncthreads();
    if (lane == 31) sums[warp] = inc;
    __syncthreads();
    int s = lane < (int)blockDim.x / 32 ? sums[lane] : 0;     // every warp scans the sums for itself
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xFFFFFFFFu, s, o);
        if (lane >= o) s += y;
    }
    total = __shfl_sync(0xFFFFFFFFu, s, 31);
    const int before = __shfl_sync(0xFFFFFFFFu, s, warp > 0 ? warp - 1 : 0);
    return (warp > 0 ? before : 0) + inc - x;
}
// Sums over the cluster's CTAs of the word at `p`: those before this one, and all.
__device__ __forceinline__ int scan_cluster(const int *p, uint32_t rank, int &total)
{
    int before = 0;
    total = 0;
    int v[kMaxPlanCtas];
#pragma unroll
    for (int c = 0; c < kMaxPlanCtas; ++c) v[c] = load_cluster(p, min(c, (int)gridDim.x - 1));      // all on their way at once
#pragma unroll
    for (int c = 0; c < kMaxPlanCtas; ++c) {
        if (c < (int)rank) before += v[c];
        if (c < (int)gridDim.x) total += v[c];
    }
    return before;
}

// The pages that thread `t` of the cluster looks after: a run of consecutive ones, so that ranks are ascending.
struct PageRun {
    int lo, hi;
    __device__ __forceinline__ PageRun(const KvArgs &a, uint32_t rank)
    {
        const int threads = gridDim.x * blockDim.x, run = (a.num_pages + threads - 1) / threads;
        const long long first = (long long)(rank * blockDim.x + threadIdx.x) * run;
        lo = (int)min(first, (long long)a.num_pages);
        hi = (int)min(first + run, (long long)a.num_pages);
    }
};

// Places that row b's next chunk covers: lo .. hi in the table, and how many more behind it.
struct Wish {
    int lo, hi, ctx;
    long long beyond;
    __device__ __forceinline__ Wish(const KvArgs &a, int b)
    {
        const int first = min(max(a.start[b], 0), a.rows), len = min(max(a.start[b + 1], first), a.rows) - first;
        ctx = max(a.ctx[b], 0);
        lo = 0;
        hi = -1;
        beyond = 0;
        if (len == 0) return;
        const long long l = (long long)ctx >> a.page_shift, h = ((long long)ctx + len - 1) >> a.page_shift;
        beyond = max(h - max(l - 1, (long long)a.width - 1), 0LL);
        lo = (int)min(l, (long long)a.width);
        hi = (int)min(h, (long long)a.width - 1);
    }
};

// A wish for page e is refused only by e's last holder among the wishes, when all holders wish: it keeps the page.  (As if
// they were served one after the other, each leaving the page unless it is the only one left.)
__device__ __forceinline__ bool takes(const KvArgs &a, const PageArgs &w, int e, unsigned long long key)
{
    if (!is_page(a, e)) return true;
    const int held = __ldcg(w.refs + e);
    return held > 1 && !(__ldcg(w.holders + e) >= held && __ldcg(w.last + e) == key);
}

__global__ void __launch_bounds__(kMaxPlanThreads)
reserve_kernel(const KvArgs a, const PageArgs w, int32_t *table, int32_t *out_missing)
{
    __shared__ int sums[32], free_here, need_here, beyond_here;
    const uint32_t rank = cluster_ctarank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int threads = blockDim.x, warps = threads / 32, ctas = gridDim.x;
    const int rows = (a.B + ctas - 1) / ctas, row0 = min((int)rank * rows, a.B), row1 = min(row0 + rows, a.B);
    pdl_wait();
    pdl_launch_dependents();
    if (rank == 0 && tid == 0) w.counts[kPageMoves] = w.counts[kPageShared] = 0;
    if (tid == 0) beyond_here = 0;
    // shared pages that are wished for: how often, and by whom last
    for (int b = row0 + warp; b < row1; b += warps) {
        const Wish wish(a, b);
        for (int i = wish.lo + lane; i <= wish.hi; i += 32) {
            const int e = table[(long long)b * a.width + i];
            if (!is_page(a, e) || w.refs[e] <= 1) continue;
            atomicAdd(w.holders + e, 1);
            atomicMax(w.last + e, ((unsigned long long)b << 32 | (uint32_t)i) + 1);
        }
    }
    const PageRun run(a, rank);
    int mine = 0;
    for (int p = run.lo; p < run.hi; ++p) mine += w.refs[p] <= 0;
    int total;
    const int free_before = scan_cta(mine, sums, total);
    if (tid == 0) free_here = total;
    cluster_sync_all();
    // pages that every row takes, and their sums
    int base = 0;
    for (int chunk = row0; chunk < row1; chunk += threads) {
        for (int b = chunk + warp; b < min(chunk + threads, row1); b += warps) {
            const Wish wish(a, b);
            int n = 0;
            for (int i = wish.lo + lane; i <= wish.hi; i += 32)
                n += takes(a, w, table[(long long)b * a.width + i], ((unsigned long long)b << 32 | (uint32_t)i) + 1);
            n = __reduce_add_sync(0xFFFFFFFFu, n);
            if (lane == 0) {
                w.row_first[b] = n;
                if (wish.beyond) atomicAdd(&beyond_here, (int)min(wish.beyond, 16384LL));    // 65535 rows stay within 31 bits
            }
        }
        __syncthreads();
        const int b = chunk + tid, n = b < row1 ? w.row_first[b] : 0;
        const int before = scan_cta(n, sums, total);
        if (b < row1) w.row_first[b] = base + before;
        base += total;
    }
    __syncthreads();
    if (tid == 0) need_here = base;
    cluster_sync_all();
    int need, beyond, free_pages;
    const int need_first = scan_cluster(&need_here, rank, need);
    scan_cluster(&beyond_here, rank, beyond);
    int at = scan_cluster(&free_here, rank, free_pages) + free_before;
    const long long missing = (long long)beyond + max(need - free_pages, 0);
    for (int p = run.lo; p < run.hi && at < need && missing == 0; ++p)
        if (w.refs[p] <= 0) w.list[at++] = p;
    cluster_sync_all();
    for (int b = row0 + warp; b < row1; b += warps) {
        const Wish wish(a, b);
        int next = need_first + w.row_first[b];
        for (int i0 = wish.lo; i0 <= wish.hi; i0 += 32) {
            const int i = i0 + lane;
            const unsigned long long key = ((unsigned long long)b << 32 | (uint32_t)i) + 1;
            const bool in = i <= wish.hi;
            int32_t *place = table + (long long)b * a.width + (in ? i : wish.lo);
            const int e = in ? *place : -1;
            const bool take = in && takes(a, w, e, key);
            // whoever wished last for a shared page has its count put right, below
            if (in && is_page(a, e) && __ldcg(w.last + e) == key) w.map[atomicAdd(w.counts + kPageShared, 1)] = e;
            const unsigned m = __ballot_sync(0xFFFFFFFFu, take);
            if (take && missing == 0) {
                const int r = next + __popc(m & ((1u << lane) - 1));
                if (debug_check(r >= 0 && r < a.num_pages, a.status, 80)) {
                    const int p = __ldcg(w.list + r);
                    *place = p;
                    w.refs[p] = 1;
                    if (is_page(a, e) && ((long long)i << a.page_shift) < wish.ctx) {
                        const int m2 = atomicAdd(w.counts + kPageMoves, 1);
                        w.from[m2] = e;
                        w.to[m2] = p;
                    }
                }
            }
            next += __popc(m);
        }
    }
    cluster_sync_all();
    const int shared = __ldcg(w.counts + kPageShared);
    for (int j = rank * threads + tid; j < shared; j += ctas * threads) {
        const int e = __ldcg(w.map + j), wished = __ldcg(w.holders + e), held = __ldcg(w.refs + e);
        if (missing == 0) w.refs[e] = max(held - wished, 1);
        w.holders[e] = 0;
        w.last[e] = 0;
    }
    if (rank == 0 && tid == 0) *out_missing = (int)min(missing, 2147483647LL);
}

// Used pages behind the first `used` places go, in ascending order, to the free ones below.
__global__ void __launch_bounds__(kMaxPlanThreads)
compact_kernel(const KvArgs a, const PageArgs w, int32_t *out_used)
{
    __shared__ int sums[32], used_here, below_here;
    const uint32_t rank = cluster_ctarank();
    const int tid = threadIdx.x;
    pdl_wait();
    pdl_launch_dependents();
    const PageRun run(a, rank);
    int mine = 0, total, used;
    for (int p = run.lo; p < run.hi; ++p) mine += w.refs[p] > 0;
    int before = scan_cta(mine, sums, total);
    if (tid == 0) used_here = total;
    cluster_sync_all();
    before += scan_cluster(&used_here, rank, used);
    mine = 0;
    for (int p = run.lo; p < min(run.hi, used); ++p) mine += w.refs[p] > 0;
    scan_cta(mine, sums, total);
    if (tid == 0) below_here = total;
    cluster_sync_all();
    int below;
    scan_cluster(&below_here, rank, below);
    for (int p = run.lo; p < run.hi; ++p) {
        const bool is_used = w.refs[p] > 0;
        if (p < used && !is_used) {
            w.to[p - before] = p;
        } else if (p >= used) {
            w.map[p] = is_used ? before - below : -1;
            if (is_used) w.from[before - below] = p;
        }
        before += is_used;
    }
    if (rank == 0 && tid == 0) {
        w.counts[kPageMoves] = used - below;
        w.counts[kPageUsed] = used;
        *out_used = used;
    }
    cluster_sync_all();                                       // the others may still read this CTA's sums
}

// ---- moving ----------------------------------------------------------------------------------------------------
// Copies page from[j] to to[j] in every layer, keys and values.  compacted: the plan is compact_kernel()'s, and counts and tables
// follow.  No page is both read and written.
__global__ void __launch_bounds__(kMoveThreads)
move_kernel(const KvArgs a, const PageArgs w, int32_t *__restrict__ table, int compacted, long long chunk, int pieces)
{
    pdl_wait();
    pdl_launch_dependents();
    const int moves = w.counts[kPageMoves];
    if (compacted && moves > 0) {
        const int used = w.counts[kPageUsed];
        const long long step = (long long)gridDim.x * kMoveThreads, me = (long long)blockIdx.x * kMoveThreads + threadIdx.x;
        for (long long i = me; i < (long long)a.B * a.width; i += step) {
            const int e = table[i];
            if (e < used || e >= a.num_pages) continue;
            const int j = w.map[e];
            if (j >= 0) table[i] = w.to[j];
        }
        for (long long j = me; j < moves; j += step) {
            w.refs[w.to[j]] = w.refs[w.from[j]];
            w.refs[w.from[j]] = 0;
        }
    }
    const long long units = (long long)moves * a.layers * 2 * pieces;
    for (long long u = blockIdx.x; u < units; u += gridDim.x) {
        const int piece = (int)(u % pieces);
        const long long rest = u / pieces;
        const bool is_v = rest & 1;
        const int layer = (int)((rest >> 1) % a.layers), j = (int)((rest >> 1) / a.layers);
        const int pf = w.from[j], pt = w.to[j];
        if (!debug_check(is_page(a, pf) && is_page(a, pt), a.status, 81)) continue;
        const long long src = (long long)layer * a.num_pages + pf, dst = (long long)layer * a.num_pages + pt;
        uint8_t *pages = static_cast<uint8_t *>(is_v ? a.v : a.k);
        const long long first = (long long)piece * kMoveBytes;
        const uint32_t bytes = (uint32_t)min(chunk - first, (long long)kMoveBytes);
        const uint4 *from = reinterpret_cast<const uint4 *>(pages + src * chunk + first);
        uint4 *to = reinterpret_cast<uint4 *>(pages + dst * chunk + first);
        uint4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((threadIdx.x + i * kMoveThreads) * 16 < bytes) x[i] = from[threadIdx.x + i * kMoveThreads];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((threadIdx.x + i * kMoveThreads) * 16 < bytes) to[threadIdx.x + i * kMoveThreads] = x[i];
        if (a.k_exps) {                                       // one byte for each d bytes of the piece
            uint8_t *exps = is_v ? a.v_exps : a.k_exps;
            const long long e_chunk = chunk / a.d, e_first = first / a.d;
            if (threadIdx.x * 16 < bytes / a.d)
                reinterpret_cast<uint4 *>(exps + dst * e_chunk + e_first)[threadIdx.x] =
                    reinterpret_cast<const uint4 *>(exps + src * e_chunk + e_first)[threadIdx.x];
        }
    }
}

// A cluster of large CTAs to plan with, or one small CTA, whose barriers take a quarter of the time, where that has little to look through
// (eight copies of a prompt made, their places reserved and all given back: 20.7 us with the cluster, 19.2 without).
template <typename... KArgs, typename... Args>
cudaError_t launch_plan(void (*kernel)(KArgs...), const KvArgs &a, cudaStream_t stream, Args &&...args)
{
    const bool small = a.num_pages <= 4096 && a.B <= 64;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = small ? 1 : kMaxPlanCtas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.gridDim = dim3(small ? 1 : kMaxPlanCtas);
    cfg.blockDim = dim3(small ? 256 : kMaxPlanThreads);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

cudaError_t launch_move(const KvArgs &a, const PageArgs &w, int32_t *table, int compacted, int sms, cudaStream_t stream)
{
    const long long chunk = (long long)a.heads * a.d * (a.k_exps ? 1 : 2) << a.page_shift;
    const int pieces = (int)((chunk + kMoveBytes - 1) / kMoveBytes);
    return launch_dependent(move_kernel, dim3(sms * 8), dim3(kMoveThreads), 0, stream, a, w, table, compacted, chunk, pieces);
}

}  // namespace

cudaError_t launch_kv_fork(const KvArgs &a, int32_t *refs, int32_t *table, int32_t *ctx, const int32_t *parent, cudaStream_t stream)
{
    return launch_dependent(fork_kernel, dim3(a.B), dim3(kRowThreads), 0, stream, a, refs, table, ctx, parent);
}

cudaError_t launch_kv_release(const KvArgs &a, int32_t *refs, int32_t *table, const int32_t *keep, cudaStream_t stream)
{
    return launch_dependent(release_kernel, dim3(a.B), dim3(kRowThreads), 0, stream, a, refs, table, keep);
}

cudaError_t launch_kv_reserve(const KvArgs &a, const PageArgs &w, int32_t *table, int32_t *out_missing, int sms, cudaStream_t stream)
{
    const cudaError_t e = launch_plan(reserve_kernel, a, stream, a, w, table, out_missing);
    return e != cudaSuccess ? e : launch_move(a, w, table, 0, sms, stream);
}

cudaError_t launch_kv_compact(const KvArgs &a, const PageArgs &w, int32_t *table, int32_t *out_used, int sms, cudaStream_t stream)
{
    const cudaError_t e = launch_plan(compact_kernel, a, stream, a, w, out_used);
    return e != cudaSuccess ? e : launch_move(a, w, table, 1, sms, stream);
}

}  // namespace dresd
