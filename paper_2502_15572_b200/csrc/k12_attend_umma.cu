// K12 -- attention of many rows per key/value head over the paged cache (drafts, pieces of a prompt), on tcgen05.
//
// One pass with the running maximum, as in K11, but every key and value meets 128 or 256 rows, so the bound is the
// tensor cores together with the exponentials (a 128 x 128 tile of scores is 512 cycles of each product at d = 128 and
// 1024 cycles of the 16 exponentials per cycle that an SM has).  A CTA (one per SM) runs TWO STREAMS of tiles, each
// with scores S, weights P and sums O of its own in TMEM (S 128 columns, P in S's place, O d columns), so that the
// tensor cores work on one stream while the other's warps take exponentials:
//
//     S_w = Q_w K^T        128 rows x 128 positions, operands in shared memory (128-byte swizzle, K-major)
//     P_w = 2^(scale S_w - m)        a thread owns a row: no shuffles; 16 bits, back to TMEM
//     O_w += P_w V         P from TMEM, V as stored ([position][d] is the MN-major operand)
//
// Items of more than 128 rows give the streams two row tiles and every loaded tile of positions to both; items of
// up to 128 rows give both streams the same rows and every second tile each, and join them at the end.  Rows of a group of heads are
// packed: 128 / group tokens x group heads are one row tile, which one TMA box of the queries fetches.
//
// Roles: warp 0 loads tiles (a lane per page and slab, so that small pages are issued side by side), warp 1 issues the products,
// warp 2 loads queries, warp 3 looks after values nobody may see (below), warps 4-7 and 8-11 are the streams' softmax;
// with an 8-bit cache warps 12-15 turn codes into 16-bit tiles.  The maximum is raised only when a score passes it by 2^8, so O
// is rarely rescaled; by then the stream's products have ended, because its next S is issued behind them.
//
// 0 x NaN is NaN, so a place that a row does not see must not reach the second product: places behind the sequence's end
// are cleared in shared memory, and non-finite values of the chunk itself are taken out there and put back at the end as
// what they make of a result, NaN, for the rows and elements that see them.
#include "kv_plan.cuh"

namespace dresd {
namespace {

constexpr int kTile = 128;                                 // rows of a row tile, positions of a tile
constexpr int kSlabBytes = kTile * 128;                    // 64 elements of every row of a tile
constexpr float kSlack = 8.f;

template <bool Q8, int D>
struct Geometry {
    static constexpr int kSlabs = D / 64;
    static constexpr int kTileBytes = kSlabs * kSlabBytes;
    static constexpr int kStages = (D == 128 ? 1 : 2) * (Q8 ? 3 : 5);     // 16-bit tiles
    static constexpr int kRaw = Q8 ? (D == 128 ? 4 : 8) : 0;              // 8-bit tiles
    static constexpr int kRawBytes = kTile * D;
    static constexpr int kThreads = Q8 ? 512 : 384;
    static constexpr int kBig = 2 * kTileBytes + kStages * kTileBytes + kRaw * kRawBytes;
    static constexpr int kSmall = 2048 + 1024;             // maxima and sums of both streams; barriers and plan
};
constexpr int kSmemBytes = 232448;                         // all of an SM's shared memory (one CTA per SM, by TMEM too)
constexpr int kMaxStages = 10, kMaxRaw = 8;

// Row tiles of one or two streams.
struct ManyRows {
    static __device__ __forceinline__ int per_tile(const AttendArgs &a) { return kTile / a.group; }     // tokens of a stream
    static __device__ __forceinline__ int row_tiles(const AttendArgs &a, const Chunk &k)
    {
        const int t = 2 * per_tile(a);
        return (k.len + t - 1) / t;
    }
    static __device__ __forceinline__ int tokens(const AttendArgs &a, const Chunk &k, int r)
    {
        const int t = 2 * per_tile(a);
        return min(t, k.len - r * t);
    }
    static __device__ __forceinline__ bool one_tile(const AttendArgs &a, const Chunk &k, int r) { return tokens(a, k, r) <= per_tile(a); }
    // position tiles that the item's rows see
    static __device__ __forceinline__ int tiles(const AttendArgs &a, const Chunk &k, int r)
    {
        int seen = k.total;
        if (!a.mask) seen = min(seen, k.ctx + r * 2 * per_tile(a) + tokens(a, k, r));
        return max(1, (seen + kTile - 1) / kTile);
    }
    // a unit keeps both streams busy for one tile: one tile of positions for two row tiles, two for one
    static __device__ __forceinline__ int units(const AttendArgs &a, const Chunk &k, int r)
    {
        const int t = tiles(a, k, r);
        return one_tile(a, k, r) ? (t + 1) / 2 : t;
    }
};

struct Shared {
    uint64_t full[kMaxStages], empty[kMaxStages], v_ok[kMaxStages];
    uint64_t raw_full[kMaxRaw], raw_empty[kMaxRaw];
    uint64_t q_full[2], q_empty[2], s_full[2], p_full[2], o_full[2];
    uint32_t tmem;
    unsigned ticket;
    int bad;                                               // a value of some chunk was not finite
    // the softmax warps' place in the plan lives here, not in their registers, which the scores need
    KvPlan<ManyRows> plan;
    Segment seg;
    int more;
};
static_assert(sizeof(Shared) <= 1024, "barriers and plan");

// What every role knows of a segment.
struct Work {
    bool one;            // both streams on the same rows
    int t0, nt;          // first position tile, tiles
    int n[2];            // tiles of the streams
    __device__ __forceinline__ Work(const AttendArgs &a, const Chunk &c, const Segment &s)
    {
        one = ManyRows::one_tile(a, c, s.rt);
        const int all = ManyRows::tiles(a, c, s.rt);
        t0 = one ? 2 * s.kt0 : s.kt0;
        nt = (one ? min(2 * s.kt1, all) : s.kt1) - t0;
        n[0] = one ? (nt + 1) / 2 : nt;
        n[1] = one ? nt / 2 : nt;
    }
    // Places of key tile j and value tile j in the order in which tiles are loaded and consumed:
    // K0 V0 K1 V1 ... for two row tiles, K0 K1 V0 K2 V1 K3 ... for one.
    __device__ __forceinline__ int k_place(int j) const { return one ? (j < 2 ? j : 2 * j - 1) : 2 * j; }
    __device__ __forceinline__ int v_place(int j) const { return one ? (j == nt - 1 ? 2 * nt - 1 : 2 + 2 * j) : 2 * j + 1; }
};

__device__ __forceinline__ void tma_load_3d(void *dst, const CUtensorMap *map, int x, int y, int z, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
        : "memory");
}
// First operand from TMEM.
__device__ __forceinline__ void umma_f16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// MN-major operand, 128-byte swizzle: 64 elements of 8 positions are 1024 bytes; the next 8 positions
// follow at once, the next 64 elements one slab on.
__device__ __forceinline__ uint64_t make_desc_mn(uint32_t smem_addr)
{
    return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | ((uint64_t)(kSlabBytes >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t *r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t *r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
// A warpgroup's registers per thread.  The warpgroups' shares together are what the CTA was launched with: 512 x 128
// (8-bit: 64 + 192 + 192 + 64 a thread of each) or 384 x 168 (88 + 208 + 208).
template <bool kMore, int kCount>
__device__ __forceinline__ void set_registers()
{
    if constexpr (kMore) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kCount));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kCount));
}
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Parts of shared items: two slots per CTA; sums as [d / 4][256 rows] float4 (a warp's rows side by side), maxima,
// weight sums, and whether a value was not finite.
constexpr int kPartRows = 2 * kTile;
__host__ __device__ constexpr size_t part_floats(int d) { return (size_t)kPartRows * (d + 2) + 32; }

// The rows of the chunk's own tokens that (row's token, j) ...: does token `tok` of the chunk see its place j?
__device__ __forceinline__ bool sees(const AttendArgs &a, const Chunk &c, int tok, int j)
{
    if (c.ctx + j >= c.total) return false;
    if (!a.mask) return j <= tok;
    return (j >> 5) < a.mask_words && (a.mask[(long long)(c.row0 + tok) * a.mask_words + (j >> 5)] >> (j & 31) & 1);
}

template <typename T, bool Q8, int D>
__global__ void __launch_bounds__(Geometry<Q8, D>::kThreads, 1)
attend_umma_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                   const __grid_constant__ CUtensorMap v_map, const AttendArgs a)
{
    using Geo = Geometry<Q8, D>;
    constexpr int kStages = Geo::kStages, kSlabs = Geo::kSlabs, kTileBytes = Geo::kTileBytes;
    extern __shared__ uint8_t smem_raw[];
    const int pad = (int)(-smem_u32(smem_raw) & 1023u);
    uint8_t *q_s = smem_raw + pad;
    uint8_t *stages = q_s + 2 * kTileBytes;
    uint8_t *raws = stages + kStages * kTileBytes;
    float *s_m = reinterpret_cast<float *>(raws + Geo::kRaw * Geo::kRawBytes);       // [2][128]
    float *s_l = s_m + 2 * kTile;                                                     // [2][128]
    Shared &sh = *reinterpret_cast<Shared *>(s_l + 2 * kTile);
    if (pad + Geo::kBig + Geo::kSmall > kSmemBytes) {       // shared memory never starts there
        if (threadIdx.x == 0) report_timeout(a.kv.status);
        return;
    }
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long wl = a.wait_cycles > 0 ? a.wait_cycles : kWaitCycles;

    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sh.full[s], Q8 ? 4 : 1);
            mbar_init(&sh.empty[s], 1);
            mbar_init(&sh.v_ok[s], 1);
        }
        for (int s = 0; s < Geo::kRaw; ++s) {
            mbar_init(&sh.raw_full[s], 1);
            mbar_init(&sh.raw_empty[s], 4);
        }
        for (int w = 0; w < 2; ++w) {
            mbar_init(&sh.q_full[w], 1);
            mbar_init(&sh.q_empty[w], 1);
            mbar_init(&sh.s_full[w], 1);
            mbar_init(&sh.p_full[w], 4);
            mbar_init(&sh.o_full[w], 1);
        }
        sh.bad = sh.more = 0;
        mbar_fence_init();
    }
    if (warp == 3) {
        tmem_alloc(&sh.tmem, 512);
        tmem_relinquish();
    }
    KvPlan<ManyRows> plan;
    const bool busy = plan.start(a, lane, 1);                  // the same for the whole CTA
    if (tid == 0) sh.plan = plan;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;                          // S0, S1 at 0, 128; O0, O1 at 256, 256 + D
    Segment seg;

    if (!busy) {
        // nothing to do: fall through to the end
    } else if (warp < 4) {
        set_registers<false, Q8 ? 64 : 88>();
        if (warp == 0) {
            // ---- tiles of keys and values: 16-bit ones straight into the stages, 8-bit ones into the raw ring
            constexpr int kRing = Q8 ? Geo::kRaw : kStages;
            constexpr int kBytes = Q8 ? Geo::kRawBytes : kTileBytes;
            constexpr int kParts = Q8 ? 1 : kSlabs;              // copies per page
            uint8_t *ring = Q8 ? raws : stages;
            uint64_t *full = Q8 ? sh.raw_full : sh.full, *empty = Q8 ? sh.raw_empty : sh.empty;
            if (lane == 0) {
                tma_prefetch_desc(&k_map);
                tma_prefetch_desc(&v_map);
            }
            const int per = kTile >> a.kv.page_shift;            // pages per tile
            const int beyond = (int)min((long long)a.kv.layers * a.kv.num_pages * a.kv.heads << a.kv.page_shift, 2147483647LL);
            int it = 0, issued = 0;
            bool ok = true;
            while (ok && plan.next(a, seg)) {
                const Chunk c = plan.c;
                const Work w(a, c, seg);
                // page of this lane's copy of tile t, as a row of the maps (out of range: zeros are loaded)
                auto row_of = [&](int t) {
                    const int p = t * kTile + ((lane / kParts) << a.kv.page_shift);
                    int page = -1;
                    if (lane < per * kParts && p < c.total)
                        page = __ldg(a.kv.table + (long long)seg.b * a.kv.width + (p >> a.kv.page_shift));
                    if (page < 0 || page >= a.kv.num_pages) return beyond;
                    return (int)kv_row(a.kv, a.kv.layer, page, seg.head, 0);
                };
                auto load = [&](const CUtensorMap *map, int row) {
                    const int s = it % kRing;
                    if (it >= kRing && !mbar_wait(&empty[s], ((it / kRing) - 1) & 1, wl)) ok = false;
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) return;
                    if (lane == 0) mbar_arrive_expect_tx(&full[s], (uint32_t)kBytes);
                    __syncwarp();
                    if (lane < per * kParts && !(a.lose_stage > 0 && blockIdx.x == 0 && it == a.lose_stage - 1)) {
                        const int pg = lane / kParts, part = lane % kParts;
                        uint8_t *dst = ring + (size_t)s * kBytes + part * kSlabBytes + ((size_t)pg << a.kv.page_shift) * (Q8 ? D : 128);
                        tma_load_2d(dst, map, part * 64, row, &full[s]);
                    }
                    ++it;
                    issued = it;
                };
                const int ahead = w.one ? 2 : 1;
                int r0 = row_of(w.t0), r1 = w.nt > 1 ? row_of(w.t0 + 1) : beyond;    // of value tiles j, j + 1
                load(&k_map, r0);
                if (ahead == 2 && w.nt > 1) load(&k_map, r1);
                for (int j = 0; j < w.nt && ok; ++j) {
                    const int r2 = j + 2 < w.nt ? row_of(w.t0 + j + 2) : beyond;
                    load(&v_map, r0);
                    if (ok && j + ahead < w.nt) load(&k_map, ahead == 2 ? r2 : r1);
                    r0 = r1;
                    r1 = r2;
                }
                plan.advance(a);
            }
            if (!ok && lane == 0) report_timeout(a.kv.status);
            // no copy may be in flight when the CTA ends
            for (int i = max(0, issued - kRing); i < issued; ++i)
                if (!mbar_wait(&full[i % kRing], (i / kRing) & 1, wl)) {
                    if (lane == 0) report_timeout(a.kv.status);
                    break;
                }
        } else if (warp == 1) {
            // ---- products
            if (lane == 0) {
                constexpr uint32_t kFmt = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
                constexpr uint32_t kCommon = (1u << 4) | (kFmt << 7) | (kFmt << 10) | ((uint32_t)(kTile >> 4) << 24);
                constexpr uint32_t kIdescS = kCommon | ((uint32_t)(kTile >> 3) << 17);
                constexpr uint32_t kIdescO = kCommon | ((uint32_t)(D >> 3) << 17) | (1u << 16);       // second operand MN-major
                int base = 0;                                    // tiles consumed by earlier segments
                int steps[2] = {0, 0}, q_uses[2] = {0, 0};
                bool ok = true;
                while (ok && plan.next(a, seg)) {
                    const Work w(a, plan.c, seg);
                    auto scores = [&](int st, int j) {
                        const int i = base + w.k_place(w.one ? 2 * j + st : j), s = i % kStages;
                        if (!mbar_wait(&sh.full[s], (i / kStages) & 1, wl)) return false;
                        tc_fence_after();
                        const uint32_t qa = smem_u32(q_s) + (w.one ? 0 : st * kTileBytes), ka = smem_u32(stages) + s * kTileBytes;
#pragma unroll
                        for (int k = 0; k < D / 16; ++k)
                            umma_f16(tmem + st * kTile, make_desc(qa + (k >> 2) * kSlabBytes) + 2 * (k & 3),
                                     make_desc(ka + (k >> 2) * kSlabBytes) + 2 * (k & 3), kIdescS, k != 0);
                        tc_commit(&sh.s_full[st]);
                        if (w.one || st == 1) tc_commit(&sh.empty[s]);
                        if (w.one ? 2 * j + st == w.nt - 1 : j == w.nt - 1) tc_commit(&sh.q_empty[w.one ? 0 : st]);
                        return true;
                    };
                    for (int st = 0; st < (w.one ? 1 : 2) && ok; ++st) {
                        ok = mbar_wait(&sh.q_full[st], q_uses[st] & 1, wl);
                        ++q_uses[st];
                    }
                    for (int st = 0; st < 2 && ok; ++st)
                        if (w.n[st] > 0) ok = scores(st, 0);
                    for (int j = 0; j < w.n[0] && ok; ++j)
                        for (int st = 0; st < 2 && ok; ++st) {
                            if (j >= w.n[st]) continue;
                            const int i = base + w.v_place(w.one ? 2 * j + st : j), s = i % kStages;
                            ok = mbar_wait(Q8 ? &sh.full[s] : &sh.v_ok[s], (i / kStages) & 1, wl) && mbar_wait(&sh.p_full[st], steps[st] & 1, wl);
                            if (!ok) break;
                            ++steps[st];
                            tc_fence_after();
                            const uint32_t va = smem_u32(stages) + s * kTileBytes;
#pragma unroll
                            for (int k = 0; k < kTile / 16; ++k)
                                umma_f16_ta(tmem + 256 + st * D, tmem + st * kTile + 8 * k, make_desc_mn(va) + 128 * k, kIdescO, (j | k) != 0);
                            if (w.one || st == 1) tc_commit(&sh.empty[s]);
                            if (j == w.n[st] - 1) tc_commit(&sh.o_full[st]);
                            else ok = scores(st, j + 1);
                        }
                    base += 2 * w.nt;
                    plan.advance(a);
                }
                if (!ok) report_timeout(a.kv.status);
            }
        } else if (warp == 2) {
            // ---- queries
            if (lane == 0) {
                tma_prefetch_desc(&q_map);
                const int tokens = ManyRows::per_tile(a);
                const uint32_t bytes = (uint32_t)(tokens * a.group * 128 * kSlabs);
                int uses[2] = {0, 0}, last[2] = {-1, -1};
                bool ok = true;
                while (ok && plan.next(a, seg)) {
                    const Work w(a, plan.c, seg);
                    for (int st = 0; st < (w.one ? 1 : 2) && ok; ++st) {
                        if (uses[st] > 0) ok = mbar_wait(&sh.q_empty[st], (uses[st] - 1) & 1, wl);
                        if (!ok) break;
                        mbar_arrive_expect_tx(&sh.q_full[st], bytes);
                        for (int p = 0; p < kSlabs; ++p)
                            tma_load_3d(q_s + st * kTileBytes + p * kSlabBytes, &q_map, p * 64, seg.head * a.group,
                                        plan.c.row0 + (2 * seg.rt + st) * tokens, &sh.q_full[st]);
                        last[st] = uses[st]++;
                    }
                    plan.advance(a);
                }
                if (!ok) report_timeout(a.kv.status);
                for (int st = 0; st < 2; ++st)
                    if (last[st] >= 0 && !mbar_wait(&sh.q_full[st], last[st] & 1, wl)) report_timeout(a.kv.status);
            }
        } else if (warp == 3) {
            // ---- values nobody may see (16-bit cache; the conversion does it for codes)
            if constexpr (!Q8) {
                constexpr uint32_t kInf = std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u;
                int base = 0;
                bool ok = true;
                while (ok && plan.next(a, seg)) {
                    const Chunk c = plan.c;
                    const Work w(a, c, seg);
                    for (int x = 0, vj = 0; x < 2 * w.nt && ok; ++x) {
                        const int i = base + x, s = i % kStages;
                        ok = __all_sync(0xFFFFFFFFu, mbar_wait(&sh.full[s], (i / kStages) & 1, wl));
                        if (!ok) break;
                        if (x == w.v_place(vj)) {
                            const int p0 = (w.t0 + vj) * kTile;
                            ++vj;
                            if (p0 + kTile > c.ctx) {
                                const int end = min(max(c.total - p0, 0), kTile);             // rows in use
                                uint4 *tile = reinterpret_cast<uint4 *>(stages + (size_t)s * kTileBytes);
                                for (int y = lane; y < kSlabs * (kTile - end) * 8; y += 32) {
                                    const int rows = kTile - end;
                                    tile[(y / (rows * 8)) * (kTile * 8) + end * 8 + y % (rows * 8)] = make_uint4(0, 0, 0, 0);
                                }
                                const int from = max(c.ctx - p0, 0), n = max(end - from, 0);
                                bool odd = false;
#pragma unroll 4
                                for (int y = lane; y < kSlabs * n * 8; y += 32) {
                                    const uint4 v = tile[(y / (n * 8)) * (kTile * 8) + from * 8 + y % (n * 8)];
                                    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                                    for (int k = 0; k < 4; ++k) odd |= (u[k] & kInf) == kInf || (u[k] >> 16 & kInf) == kInf;
                                }
                                if (__any_sync(0xFFFFFFFFu, odd)) {
                                    for (int y = lane; y < kSlabs * n * 8; y += 32) {
                                        uint32_t *u = reinterpret_cast<uint32_t *>(&tile[(y / (n * 8)) * (kTile * 8) + from * 8 + y % (n * 8)]);
                                        for (int k = 0; k < 4; ++k) {
                                            if ((u[k] & kInf) == kInf) u[k] &= 0xFFFF0000u;
                                            if ((u[k] >> 16 & kInf) == kInf) u[k] &= 0x0000FFFFu;
                                        }
                                    }
                                    *reinterpret_cast<volatile int *>(&sh.bad) = 1;
                                }
                                fence_async_smem();
                                __syncwarp();
                            }
                        }
                        if (lane == 0) mbar_arrive(&sh.v_ok[s]);
                    }
                    base += 2 * w.nt;
                    plan.advance(a);
                }
                if (!ok && lane == 0) report_timeout(a.kv.status);
            }
        }
    } else if (warp < 12) {
        set_registers<true, Q8 ? 192 : 208>();
        // ---- softmax of stream st; a thread owns a row
        const int st = warp >= 8 ? 1 : 0;
        const int row = tid & 127;                           // TMEM lane
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;    // (warp % 4) x 32 lanes, in the address's upper half
        const uint32_t ts = tmem + lanes + st * kTile, to = tmem + lanes + 256 + st * D;
        const int per = ManyRows::per_tile(a);
        const int heads = a.kv.heads * a.group;
        const float scale = a.scale_log2;
        int steps = 0, items[2] = {0, 0};
        bool dead = false;
        while (true) {
            bar_sync(1, 256);                                // the last segment's readers are done (O, s_m, s_l too)
            if (tid == 128) {
                if (sh.more) sh.plan.advance(a);
                sh.more = sh.plan.next(a, sh.seg);
            }
            bar_sync(1, 256);
            if (!sh.more) break;
            const Work w(a, sh.plan.c, sh.seg);
            const Segment &seg = sh.seg;
            const Chunk &c = sh.plan.c;
            const int first_tok = (2 * seg.rt + (w.one ? 0 : st)) * per;
            const int tok = first_tok + row / a.group;       // of this row; may lie behind the chunk
            const bool valid = row < per * a.group && tok < c.len;
            const int limit = a.mask ? c.total : min(c.total, c.ctx + min(tok, c.len - 1) + 1);
            const int all_seen = min(c.total, a.mask ? c.ctx : c.ctx + min(first_tok, c.len - 1) + 1);    // by every row
            const uint32_t *mask = a.mask ? a.mask + (long long)(c.row0 + min(tok, c.len - 1)) * a.mask_words : nullptr;
            float m = -INFINITY, l = 0.f;
            for (int j = 0; j < w.n[st]; ++j) {
                const int p0 = (w.t0 + (w.one ? 2 * j + st : j)) * kTile;
                if (!dead && !mbar_wait(&sh.s_full[st], steps & 1, wl)) {
                    report_timeout(a.kv.status);
                    dead = true;
                }
                dead = __any_sync(0xFFFFFFFFu, dead);
                ++steps;
                tc_fence_after();
                float s[kTile];
#pragma unroll
                for (int k = 0; k < kTile; k += 32) tmem_ld32(ts + k, reinterpret_cast<uint32_t *>(s) + k);
                tmem_ld_wait();
                if (p0 + kTile > all_seen) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int p = p0 + 32 * k;
                        const int n = min(max(limit - p, 0), 32);
                        uint32_t see = n == 32 ? 0xFFFFFFFFu : (1u << n) - 1u;
                        if (a.mask && p + 32 > c.ctx) {
                            const int j0 = p - c.ctx;         // place in the chunk of bit 0; context below 0
                            const int w0 = j0 >> 5;           // floor
                            const uint32_t lo = w0 >= 0 && w0 < a.mask_words ? mask[w0] : w0 < 0 ? 0xFFFFFFFFu : 0u;
                            const uint32_t hi = w0 + 1 >= 0 && w0 + 1 < a.mask_words ? mask[w0 + 1] : 0u;
                            see &= __funnelshift_r(lo, hi, j0 & 31);
                        }
#pragma unroll
                        for (int x = 0; x < 32; ++x)
                            if (!(see >> x & 1)) s[32 * k + x] = -INFINITY;
                    }
                }
                float mx = s[0];
#pragma unroll
                for (int k = 1; k < kTile; ++k) mx = fmaxf(mx, s[k]);
                if (__any_sync(0xFFFFFFFFu, (mx - m) * scale > kSlack)) {     // -inf - -inf is NaN: no
                    const float mn = fmaxf(m, mx);
                    if (j > 0) {
                        const float f = mn > -INFINITY ? ex2((m - mn) * scale) : 1.f;
                        l *= f;
#pragma unroll 1
                        for (int k = 0; k < D; k += 16) {
                            uint32_t r[16];
                            tmem_ld16(to + k, r);
                            tmem_ld_wait();
#pragma unroll
                            for (int x = 0; x < 16; ++x) r[x] = __float_as_uint(__uint_as_float(r[x]) * f);
                            tmem_st16(to + k, r);
                        }
                    }
                    m = mn;
                }
                const float base = m > -INFINITY ? m * scale : 0.f;
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c0 = 0; c0 < kTile; c0 += 32) {       // in pieces, so that scores leave the registers as weights come
                    uint32_t p[16];
#pragma unroll
                    for (int k = 0; k < 32; k += 2) {
                        const float x = ex2(fmaf(s[c0 + k], scale, -base)), y = ex2(fmaf(s[c0 + k + 1], scale, -base));
                        sum[k / 2 % 2 * 2] += x;
                        sum[k / 2 % 2 * 2 + 1] += y;
                        p[k / 2] = pack2<T>(x, y);
                    }
                    tmem_st16(ts + c0 / 2, p);
                }
                l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.p_full[st]);
            }
            // ---- the segment's result
            s_m[st * kTile + row] = m;
            s_l[st * kTile + row] = l;
            for (int x = 0; x < 2; ++x)
                if (w.n[x] > 0) {
                    if ((w.one || x == st) && !dead && !mbar_wait(&sh.o_full[x], items[x] & 1, wl)) {
                        report_timeout(a.kv.status);
                        dead = true;
                    }
                    ++items[x];
                }
            dead = __any_sync(0xFFFFFFFFu, dead);
            tc_fence_after();
            bar_sync(1, 256);
            // rows and elements of this thread: two row tiles: row 128 st + row, all elements; one: row `row`, half of them,
            // from both streams
            const int d0 = w.one ? st * (D / 2) : 0, d1 = w.one ? d0 + D / 2 : D;
            const int prow = w.one ? row : st * kTile + row;
            float f0 = 1.f, f1 = 0.f;
            if (w.one) {
                const float ma = s_m[row], mb = s_m[kTile + row];
                m = fmaxf(ma, mb);
                f0 = m > -INFINITY ? ex2((ma - m) * scale) : 0.f;
                f1 = m > -INFINITY ? ex2((mb - m) * scale) : 0.f;
                l = f0 * s_l[row] + f1 * s_l[kTile + row];
            }
            const bool split = seg.c0 != seg.c1;
            const long long at = (long long)(c.row0 + tok) * heads + seg.head * a.group + row % a.group;
            bool bad = *reinterpret_cast<volatile int *>(&sh.bad) != 0;
            auto put = [&](int d, const float *x, float inv) {       // 32 elements of the result
                if (!valid) return;
                uint4 *dst = reinterpret_cast<uint4 *>(static_cast<T *>(a.out) + at * D + d);
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    dst[v] = make_uint4(pack2<T>(x[8 * v] * inv, x[8 * v + 1] * inv), pack2<T>(x[8 * v + 2] * inv, x[8 * v + 3] * inv),
                                        pack2<T>(x[8 * v + 4] * inv, x[8 * v + 5] * inv), pack2<T>(x[8 * v + 6] * inv, x[8 * v + 7] * inv));
            };
            float *slots = a.part;
            float *part = slots + ((size_t)blockIdx.x * 2 + seg.slot) * part_floats(D);
            float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;       // a NaN sum stays one
#pragma unroll 1
            for (int d = d0; d < d1; d += 32) {
                uint32_t r[32];
                float x[32];
                tmem_ld32(w.one ? tmem + lanes + 256 + d : to + d, r);
                tmem_ld_wait();
#pragma unroll
                for (int k = 0; k < 32; ++k) x[k] = __uint_as_float(r[k]);
                if (w.one) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) x[k] = f0 > 0.f || f0 != f0 ? f0 * x[k] : 0.f;
                    if (w.n[1] > 0) {
                        tmem_ld32(tmem + lanes + 256 + D + d, r);
                        tmem_ld_wait();
#pragma unroll
                        for (int k = 0; k < 32; ++k) x[k] += f1 > 0.f || f1 != f1 ? f1 * __uint_as_float(r[k]) : 0.f;
                    }
                }
                if (!split) put(d, x, inv);
                else if (valid) {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        __stcg(reinterpret_cast<float4 *>(part) + (size_t)(d / 4 + k) * kPartRows + prow,
                               make_float4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]));
                }
            }
            bool done = !split;
            if (split) {
                if (d0 == 0) {
                    __stcg(part + kPartRows * D + prow, m);
                    __stcg(part + kPartRows * (D + 1) + prow, l);
                }
                if (tid == 128) __stcg(part + kPartRows * (D + 2), bad ? 1.f : 0.f);
                __threadfence();
                bar_sync(1, 256);
                if (tid == 128) sh.ticket = atomicAdd(a.tickets + seg.c0, 1u);
                bar_sync(1, 256);
                done = *reinterpret_cast<volatile unsigned *>(&sh.ticket) == (unsigned)(seg.c1 - seg.c0);
                if (done) {                                       // the last of the item's CTAs: join the parts in order
                    __threadfence();
                    if (tid == 128) a.tickets[seg.c0] = 0;
                    m = -INFINITY;
                    for (int i = seg.c0; i <= seg.c1; ++i) {
                        const float *ps = slots + ((size_t)i * 2 + (i == seg.c0 ? seg.slot0 : 0)) * part_floats(D);
                        m = fmaxf(m, __ldcg(ps + kPartRows * D + prow));
                        bad |= __ldcg(ps + kPartRows * (D + 2)) != 0.f;
                    }
                    l = 0.f;
                    for (int i = seg.c0; i <= seg.c1; ++i) {
                        const float *ps = slots + ((size_t)i * 2 + (i == seg.c0 ? seg.slot0 : 0)) * part_floats(D);
                        const float f = m > -INFINITY ? ex2((__ldcg(ps + kPartRows * D + prow) - m) * scale) : 0.f;
                        l += f * __ldcg(ps + kPartRows * (D + 1) + prow);
                    }
                    inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
#pragma unroll 1
                    for (int d = d0; d < d1; d += 32) {
                        float x[32];
#pragma unroll
                        for (int k = 0; k < 32; ++k) x[k] = 0.f;
                        for (int i = seg.c0; i <= seg.c1; ++i) {
                            const float *ps = slots + ((size_t)i * 2 + (i == seg.c0 ? seg.slot0 : 0)) * part_floats(D);
                            const float f = m > -INFINITY ? ex2((__ldcg(ps + kPartRows * D + prow) - m) * scale) : 0.f;
                            float4 y[8];
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                y[k] = valid ? __ldcg(reinterpret_cast<const float4 *>(ps) + (size_t)(d / 4 + k) * kPartRows + prow) : make_float4(0.f, 0.f, 0.f, 0.f);
                            if (f > 0.f || f != f) {
#pragma unroll
                                for (int k = 0; k < 8; ++k) {
                                    x[4 * k] += f * y[k].x;
                                    x[4 * k + 1] += f * y[k].y;
                                    x[4 * k + 2] += f * y[k].z;
                                    x[4 * k + 3] += f * y[k].w;
                                }
                            }
                        }
                        put(d, x, inv);
                    }
                }
            }
            if (done && valid) {
                if (a.lse && d0 == 0) a.lse[at] = (m > -INFINITY ? m * scale + log2f(l) : -INFINITY) * 0.69314718055994531f;
                if constexpr (!Q8) {
                    if (bad)
                        for (int t = 0; t < c.len; ++t) {
                            if (!sees(a, c, tok, t)) continue;
                            const int p = c.ctx + t;
                            int page = a.kv.table[(long long)seg.b * a.kv.width + (p >> a.kv.page_shift)];
                            if (page < 0 || page >= a.kv.num_pages) continue;
                            const T *v = static_cast<const T *>(a.kv.v) + kv_row(a.kv, a.kv.layer, page, seg.head, p & ((1 << a.kv.page_shift) - 1)) * D;
                            for (int d = d0; d < d1; ++d) {
                                const float x = unpack2<T>(*reinterpret_cast<const uint16_t *>(v + d)).x;
                                if (!isfinite(x)) reinterpret_cast<uint16_t *>(a.out)[at * D + d] = 0x7FFF;     // NaN in both types
                            }
                        }
                }
            }
            tc_fence_before();
        }
    } else {
        // ---- 8-bit tiles -> 16-bit tiles (128 threads)
        if constexpr (Q8) {
            set_registers<false, 64>();
            constexpr int kPieces = D / 16;                  // 16-byte pieces of a position
            const int t = tid & 127;
            int i = 0;                                       // tiles done
            bool ok = true;
            while (ok && plan.next(a, seg)) {
                const Chunk c = plan.c;
                const Work w(a, c, seg);
                for (int x = 0, kj = 0, vj = 0; x < 2 * w.nt && ok; ++x, ++i) {
                    const bool is_v = x == w.v_place(vj);
                    const int p0 = (w.t0 + (is_v ? vj++ : kj++)) * kTile;
                    // exponents of the positions this thread converts: t / kPieces + n x 128 / kPieces
                    int eb[kPieces];
#pragma unroll
                    for (int n = 0; n < kPieces; ++n) {
                        const int p = p0 + t / kPieces + n * (kTile / kPieces);
                        eb[n] = -1;
                        if (p < c.total) {
                            const int page = __ldg(a.kv.table + (long long)seg.b * a.kv.width + (p >> a.kv.page_shift));
                            if (page >= 0 && page < a.kv.num_pages)
                                eb[n] = (is_v ? a.kv.v_exps : a.kv.k_exps)[kv_row(a.kv, a.kv.layer, page, seg.head, p & ((1 << a.kv.page_shift) - 1))];
                        }
                    }
                    const int rs = i % Geo::kRaw, s = i % kStages;
                    bool got = mbar_wait(&sh.raw_full[rs], (i / Geo::kRaw) & 1, wl);
                    if (i >= kStages) got = got && mbar_wait(&sh.empty[s], ((i / kStages) - 1) & 1, wl);
                    ok = __all_sync(0xFFFFFFFFu, got);
                    if (!ok) break;
                    const uint8_t *raw = raws + (size_t)rs * Geo::kRawBytes;
                    uint8_t *tile = stages + (size_t)s * kTileBytes;
                    const bool clean = p0 + kTile <= c.ctx;
#pragma unroll
                    for (int n = 0; n < kPieces; ++n) {
                        const int pos = t / kPieces + n * (kTile / kPieces), piece = t % kPieces;
                        const uint4 r = *reinterpret_cast<const uint4 *>(raw + pos * D + piece * 16);
                        uint32_t u[4] = {r.x, r.y, r.z, r.w};
                        const int e = max(eb[n], 0);
                        if (!clean) {                          // unused places and the code of NaN count as 0
#pragma unroll
                            for (int k = 0; k < 4; ++k) u[k] = eb[n] < 0 ? 0u : u[k] & ~__vcmpeq4(u[k] & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
                        }
                        const uint32_t sc = scale_bits<T>(e) * 0x10001u;
                        uint32_t o[8];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            o[2 * k] = codes_to_pair<T>(__byte_perm(u[k], 0, 0x1404), sc);
                            o[2 * k + 1] = codes_to_pair<T>(__byte_perm(u[k], 0, 0x3424), sc);
                        }
                        if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                            if (e > 134) {
                                const uint32_t big = big_scale(e) * 0x10001u;
#pragma unroll
                                for (int k = 0; k < 8; ++k) {
                                    const __nv_bfloat162 y = __hmul2(*reinterpret_cast<__nv_bfloat162 *>(&o[k]), *reinterpret_cast<const __nv_bfloat162 *>(&big));
                                    o[k] = *reinterpret_cast<const uint32_t *>(&y);
                                }
                            }
                        }
                        // two 16-byte chunks of the slab's 128-byte row, swizzled by the row; every second piece stores
                        // its second chunk first, which spreads the slabs over the banks
                        uint8_t *dst = tile + (piece >> 2) * kSlabBytes + pos * 128;
                        const int ch = (piece & 3) * 2, sw = pos & 7, flip = piece >> 2 & 1;
                        *reinterpret_cast<uint4 *>(dst + (((ch + flip) ^ sw) << 4)) = flip ? make_uint4(o[4], o[5], o[6], o[7]) : make_uint4(o[0], o[1], o[2], o[3]);
                        *reinterpret_cast<uint4 *>(dst + (((ch + 1 - flip) ^ sw) << 4)) = flip ? make_uint4(o[0], o[1], o[2], o[3]) : make_uint4(o[4], o[5], o[6], o[7]);
                    }
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(&sh.full[s]);
                        mbar_arrive(&sh.raw_empty[rs]);
                    }
                }
                plan.advance(a);
            }
            if (!ok && lane == 0) report_timeout(a.kv.status);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 3) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

template <typename T, bool Q8, int D>
cudaError_t launch(const CUtensorMap &q_map, const CUtensorMap &k_map, const CUtensorMap &v_map, const AttendArgs &a, int sms,
                   cudaStream_t stream)
{
    static_assert(Geometry<Q8, D>::kBig + Geometry<Q8, D>::kSmall <= kSmemBytes, "shared memory");
    const cudaError_t e = cudaFuncSetAttribute(attend_umma_kernel<T, Q8, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    if (e != cudaSuccess) return e;
    attend_umma_kernel<T, Q8, D><<<sms, Geometry<Q8, D>::kThreads, kSmemBytes, stream>>>(q_map, k_map, v_map, a);
    return cudaGetLastError();
}

}  // namespace

size_t attend_umma_part_floats(int sms, int d) { return (size_t)sms * 2 * part_floats(d); }

cudaError_t launch_attend_umma(const CUtensorMap &q_map, const CUtensorMap &k_map, const CUtensorMap &v_map,
                               const AttendArgs &a, int sms, cudaStream_t stream)
{
    const bool q8 = a.kv.k_exps != nullptr;
    if (a.kv.dtype == kF16) {
        if (a.kv.d == 64) return q8 ? launch<__half, true, 64>(q_map, k_map, v_map, a, sms, stream) : launch<__half, false, 64>(q_map, k_map, v_map, a, sms, stream);
        return q8 ? launch<__half, true, 128>(q_map, k_map, v_map, a, sms, stream) : launch<__half, false, 128>(q_map, k_map, v_map, a, sms, stream);
    }
    if (a.kv.d == 64) return q8 ? launch<__nv_bfloat16, true, 64>(q_map, k_map, v_map, a, sms, stream) : launch<__nv_bfloat16, false, 64>(q_map, k_map, v_map, a, sms, stream);
    return q8 ? launch<__nv_bfloat16, true, 128>(q_map, k_map, v_map, a, sms, stream) : launch<__nv_bfloat16, false, 128>(q_map, k_map, v_map, a, sms, stream);
}

}  // namespace dresd
