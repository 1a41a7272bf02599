// K12 -- attention of many rows per key/value head over the paged cache (drafts, pieces of a prompt), on tcgen05.
//
// One pass with the running maximum, as in K11, but every key and value meets 128 or 256 rows, so the bound is the
// tensor cores together with the exponentials (a 128 x 128 tile of scores is 512 cycles of each product at d = 128 and
// 1024 cycles of the 16 exponentials per cycle that an SM has).  A CTA (one per SM) runs TWO STREAMS of tiles, each
// with scores S, weights P and sums O of its own in TMEM (S 128 columns, O d columns; P 64 columns, which at d = 128
// are S's, as TMEM is full), so that the tensor cores work on one stream while the other's warps take exponentials:
//
//     S_w = Q_w K^T        128 rows x 128 positions, operands in shared memory (128-byte swizzle, K-major)
//     P_w = 2^(scale S_w - m)        two threads own a row, 64 positions each: no shuffles; 16 bits, back to TMEM
//     O_w += P_w V         P from TMEM, V as stored ([position][d] is the MN-major operand)
//
// When there are fewer items than CTAs, clusters of two or four CTAs share an item: the 2 x ctas streams take every
// (2 x ctas)-th tile and send their sums through distributed shared memory, each CTA adding up its share of them.
//
// Items of more than 128 rows give the streams two row tiles and every loaded tile of positions to both; items of
// up to 128 rows give both streams the same rows and every second tile each, and join them at the end.  Rows of a group of heads are
// packed: 128 / group tokens x group heads are one row tile, which one TMA box of the queries fetches.
//
// Roles: warp 0 loads tiles (a lane per page and slab, so that small pages are issued side by side), warps 1 and 3 issue the
// products of a stream each, warp 2 works out the CTA's segments and loads their queries, warps 4-11 and 12-19 are the streams'
// softmax; with an 8-bit cache warps 20-27 turn codes into 16-bit tiles.
//
// The chain scores -> weights -> second product -> next scores of a stream is what bounds a long call (its S, P and O fill
// TMEM, so a stream has one tile in the works), hence: two threads to a row, an issuing warp to a stream; the maximum only
// raised when a score passes it by 2^8, so that O is rarely rescaled (by then the stream's products have ended, its next S is
// issued behind them); the streams' products issued in turn, so that one stream's exponentials fall into the
// other's products.
//
// Measured (148 SMs; medians): 2047 rows x 4 heads of 128 at 12345 positions, bf16, 455 us = 0.98 PFLOP/s (the power limit moves it,
// single runs take 400 to 470; the tensor cores are busy half of the time), with an 8-bit cache 531 (fp16 478); 148 items of 244 rows
// at 8000 positions, heads of 64, 118 us, with an 8-bit cache 124, the converting warps' instructions between those of the
// softmax; three drafts of twenty tokens of 16 sequences, 8 bits, 53 us; ten of ten of one sequence 23.6 us, of which at most
// three tiles a stream, some 5 us, are the chain.  Taking a quarter of the exponentials on the FMA pipes changed the first by nothing
// and cost 2 us of the second: the chain's instructions and its four handovers a tile bound it, not the exponentials' unit.
//
// 8-bit tiles become tiles of the queries' type, which holds every code x 2^e exactly: behind the conversion an 8-bit cache is a 16-bit
// one, and no row's size matters to another.
//
// 0 x NaN is NaN, so what a row does not see must not reach the second product as a non-finite number.  Places behind the
// sequence's end are cleared in shared memory.  Values of the chunk itself are not looked at unless a sum comes out
// non-finite; then repair() adds up the row again without the ones it does not see.
#include "kv_plan.cuh"

namespace dresd {
namespace {

constexpr int kTile = 128;                                 // rows of a row tile, positions of a tile
constexpr int kSlabBytes = kTile * 128;                    // 64 elements of every row of a tile
constexpr float kSlack = 8.f;
constexpr int kMaxCtas = 4;                                // of a cluster
constexpr int kConvert = 8;                                // warps that convert 8-bit tiles
// Queries and join of a segment take about as long as three tiles: 160 ragged items of 244 rows 53 us, 59 with 1, 55 with 2, 61 with 8.
constexpr int kFixed = 3;

template <bool Q8, int D>
struct Geometry {
    static constexpr int kSlabs = D / 64;
    static constexpr int kTileBytes = kSlabs * kSlabBytes;
    static constexpr int kStages = (D == 128 ? 1 : 2) * (Q8 ? 3 : 4);     // 16-bit tiles
    static constexpr int kRaw = Q8 ? (D == 128 ? 1 : 2) * 2 : 0;          // 8-bit tiles
    static constexpr int kRawBytes = kTile * D;
    static constexpr int kThreads = Q8 ? 896 : 640;
    // Two tiles of queries -- or one, and in a cluster what its CTAs send: sums (of all but a CTA itself, at most 3/4 of
    // 128 rows in fp32), maxima and weight sums -- then the rings.
    static constexpr int kMl = kMaxCtas * kTile * 8;
    static constexpr int kFront = kTileBytes + kTile * D * 4 / kMaxCtas * (kMaxCtas - 1) + kMl;
    static_assert(kFront >= 2 * kTileBytes && kFront % 1024 == 0, "room for the queries, tiles aligned");
    static constexpr int kBig = kFront + kStages * kTileBytes + kRaw * kRawBytes;
};
constexpr int kSmemBytes = 232448;                         // all of an SM's shared memory (one CTA per SM, by TMEM too)

// Row tiles of one or two streams (of one in a cluster).
struct ManyRows {
    static __device__ __forceinline__ int per_tile(const AttendArgs &a) { return a.tile_tokens; }     // tokens of a stream
    static __device__ __forceinline__ int row_tiles(const AttendArgs &a, const Chunk &k) { return a.by_rows.ceil(k.len); }
    static __device__ __forceinline__ int tokens(const AttendArgs &a, const Chunk &k, int r)
    {
        return min((int)a.by_rows.d, k.len - r * (int)a.by_rows.d);
    }
    static __device__ __forceinline__ bool one_tile(const AttendArgs &a, const Chunk &k, int r) { return tokens(a, k, r) <= per_tile(a); }
    // position tiles that the item's rows see
    static __device__ __forceinline__ int tiles(const AttendArgs &a, const Chunk &k, int r)
    {
        const int seen = a.mask ? k.total : k.upto(r * (int)a.by_rows.d + tokens(a, k, r) - 1);
        return max(1, (seen + kTile - 1) / kTile);
    }
    // a unit keeps all streams busy for one tile: one tile of positions for two row tiles, one for each stream for one
    static __device__ __forceinline__ int units(const AttendArgs &a, const Chunk &k, int r)
    {
        const int t = tiles(a, k, r);
        return one_tile(a, k, r) ? a.by_unit.ceil(t) : t;
    }
};

// What every role knows of a segment, worked out once by warp 2 and handed over in shared memory.
struct Job {
    Segment seg;
    Chunk c;
    int more;            // 0: there are no more segments
    int one;             // both streams (of every CTA of a cluster) on the same rows
    int t0, step;        // this CTA's tile j is t0 + j, or of one: t0 + j / 2 x step + j % 2
    int nt;              // its tiles
    int n[2];            // tiles of the streams
    __device__ __forceinline__ void set(const AttendArgs &a, int rank)
    {
        more = 1;
        one = ManyRows::one_tile(a, c, seg.rt);
        const int all = ManyRows::tiles(a, c, seg.rt);
        if (one) {
            step = 2 * a.ctas;
            t0 = step * seg.kt0 + 2 * rank;
            const int end = min(step * seg.kt1, all);
            n[0] = a.by_unit.ceil(max(0, end - t0));
            n[1] = a.by_unit.ceil(max(0, end - t0 - 1));
            nt = n[0] + n[1];
        } else {
            step = 2;
            t0 = seg.kt0;
            n[0] = n[1] = nt = seg.kt1 - seg.kt0;
        }
    }
    __device__ __forceinline__ int tile(int j) const { return t0 + (one ? (j >> 1) * step + (j & 1) : j); }
    // Place of value tile j in the order in which tiles are loaded and consumed: K0 V0 K1 V1 ... for two row tiles, K0 K1 V0
    // K2 V1 K3 ... for one.
    __device__ __forceinline__ int v_place(int j) const { return one ? (j == nt - 1 ? 2 * nt - 1 : 2 + 2 * j) : 2 * j + 1; }
};

template <int kStages, int kRaw>
struct Shared {
    float m[2][kTile], l[2][kTile];                        // of the streams' rows; l also passes maxima between a row's threads
    uint64_t full[kStages], empty[kStages];
    uint64_t raw_full[kRaw ? kRaw : 1], raw_empty[kRaw ? kRaw : 1];
    uint64_t q_full[2], q_empty[2], s_full[2], p_full[2], o_full[2], drained[2];
    uint64_t job_full[2], job_empty[2];
    uint64_t ready, taken;                                 // cluster: all sums have come / every CTA has read its share
    alignas(16) uint8_t exps[kRaw ? kRaw : 1][kRaw ? kTile : 16];      // exponents of the 8-bit tiles (bulk copies: 16-byte aligned)
    Job job[2];
    uint32_t tmem;
    unsigned ticket;
    unsigned tensor;                                       // 1: a stream's products are being issued
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
// Waits for the loads, and tells the compiler that these 32 registers come with it.
__device__ __forceinline__ void tmem_ld_wait_for(uint32_t *r)
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                   "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                   "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :: "memory");
}
__device__ __forceinline__ void tmem_ld_wait16(uint32_t *r)
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :: "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t *r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// A warpgroup's registers per thread.  The warpgroups' shares together are what the CTA was launched with: 640 x 96
// (64 + 4 x 104 a thread of each), with an 8-bit cache 896 x 72 (56 + 4 x 96 + 2 x 32).
template <bool kMore, int kCount>
__device__ __forceinline__ void set_registers()
{
    if constexpr (kMore) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kCount));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kCount));
}
// Barrier and "any of them".
__device__ __forceinline__ bool bar_or(int id, int threads, bool x)
{
    int r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.s32 q, %3, 0;\n\t"
        "bar.red.or.pred p, %1, %2, q;\n\t"
        "selp.s32 %0, 1, 0, p;\n\t}"
        : "=r"(r)
        : "r"(id), "r"(threads), "r"((int)x)
        : "memory");
    return r != 0;
}
__device__ __forceinline__ bool elect_one()
{
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xFFFFFFFF;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r));
    return r != 0;
}
// Parts of shared items: two slots per CTA; sums as [d / 4][256 rows] float4 (a warp's rows side by side), maxima and
// weight sums.
constexpr int kPartRows = 2 * kTile;
__host__ __device__ constexpr size_t part_floats(int d) { return (size_t)kPartRows * (d + 2); }

// Packed pairs of floats.
__device__ __forceinline__ uint64_t pair(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// Sums of stream `st` for row `row` and elements d .. d + 15 of a segment, added up one position after the other without what the
// row does not see -- called when the tensor cores' sum is not finite.  Leaves `x` alone if the chunk's own values are
// finite (then the non-finite ones are seen by every row).
template <typename T, int D>
__device__ __noinline__ void repair(const AttendArgs &a, const Job &job, int st, int row, int tok, float m, int d, float *x)
{
    const Chunk &c = job.c;
    tok = min(tok, c.len - 1);
    const int head = job.seg.head, heads = a.group, in_page = (1 << a.kv.page_shift) - 1;
    const T *q = static_cast<const T *>(a.q) + (long long)(c.row0 + tok) * a.q_row + (long long)(head * heads + row - a.by_group.div(row) * heads) * a.q_head;
    auto row_of = [&](int p) {
        if (!debug_check(p >= 0 && (p >> a.kv.page_shift) < a.kv.width, a.kv.status, 78)) p = 0;
        const int page = a.kv.table[(long long)job.seg.b * a.kv.width + (p >> a.kv.page_shift)];
        return kv_row(a.kv, a.kv.layer, page < 0 || page >= a.kv.num_pages ? 0 : page, head, p & in_page);
    };
    float y[16] = {};
    bool odd = false;
    for (int pass = 0; pass < 2; ++pass) {
        for (int j = 0; j < job.n[st]; ++j) {
            const int p0 = job.tile(job.one ? 2 * j + st : j) * kTile;
            for (int p = max(p0, pass ? 0 : c.ctx); p < min(p0 + kTile, c.total); ++p) {
                const long long r = row_of(p);
                const T *k = static_cast<const T *>(a.kv.k) + r * D, *v = static_cast<const T *>(a.kv.v) + r * D + d;
                if (pass == 0) {
                    for (int e = 0; e < 16; ++e) odd |= !isfinite(unpack2<T>(reinterpret_cast<const uint16_t *>(v)[e]).x);
                    continue;
                }
                const int t = p - c.ctx;
                if (t >= 0 && !(a.mask ? (t >> 5) < a.mask_words && (a.mask[(long long)(c.row0 + tok) * a.mask_words + (t >> 5)] >> (t & 31) & 1) : t <= tok)) continue;
                float s = 0.f;
                for (int e = 0; e < D; e += 2) {
                    const float2 kk = unpack2<T>(*reinterpret_cast<const uint32_t *>(k + e)), qq = unpack2<T>(*reinterpret_cast<const uint32_t *>(q + e));
                    s = fmaf(kk.x, qq.x, s);
                    s = fmaf(kk.y, qq.y, s);
                }
                const float w = unpack2<T>(pack2<T>(ex2(s * a.scale_log2 - m + Lift<T>::value), 0.f)).x;
                for (int e = 0; e < 16; ++e) y[e] += w * unpack2<T>(reinterpret_cast<const uint16_t *>(v)[e]).x;
            }
        }
        if (pass == 0 && !odd) return;
    }
    for (int e = 0; e < 16; ++e) x[e] = y[e];
}

template <typename T, bool Q8, int D>
__global__ void __launch_bounds__(Geometry<Q8, D>::kThreads, 1)
attend_umma_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                   const __grid_constant__ CUtensorMap v_map, const __grid_constant__ AttendArgs a)
{
    using Geo = Geometry<Q8, D>;
    using Sh = Shared<Geo::kStages, Geo::kRaw>;
    constexpr int kStages = Geo::kStages, kSlabs = Geo::kSlabs, kTileBytes = Geo::kTileBytes;
    constexpr bool kOwnP = D == 64;                         // weights have columns of their own
    constexpr int kPAt = 384;                               // then: there
    static_assert(Geo::kBig + sizeof(Sh) <= kSmemBytes, "shared memory");
    extern __shared__ uint8_t smem_raw[];
    uint8_t *q_s = smem_raw;
    float4 *sent = reinterpret_cast<float4 *>(q_s + kTileBytes);       // [other CTA][octet / CTAs][2][128 rows]
    float4 *kept = reinterpret_cast<float4 *>(q_s);        // this CTA's own share, where its queries were
    float2 *sent_ml = reinterpret_cast<float2 *>(q_s + Geo::kFront - Geo::kMl);        // [CTA][128 rows]
    uint8_t *stages = q_s + Geo::kFront;
    uint8_t *raws = stages + kStages * kTileBytes;
    Sh &sh = *reinterpret_cast<Sh *>(raws + Geo::kRaw * Geo::kRawBytes);
    if (smem_u32(smem_raw) & 1023u) {                       // shared memory never starts there
        if (threadIdx.x == 0) report_timeout(a.kv.status);
        return;
    }
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long wl = a.wait_cycles;
    const int rank = a.ctas > 1 ? (int)cluster_ctarank() : 0;

    KvPlan<ManyRows> plan;
    bool more = false;
    if (warp == 0) {
        if (lane < kStages) {
            mbar_init(&sh.full[lane], Q8 ? kConvert : 1);
            mbar_init(&sh.empty[lane], 2);                  // both streams
        }
        if (lane < Geo::kRaw) {
            mbar_init(&sh.raw_full[lane], 1);
            mbar_init(&sh.raw_empty[lane], kConvert);
        }
        if (lane < 2) {
            mbar_init(&sh.q_full[lane], 1);
            mbar_init(&sh.q_empty[lane], lane == 0 && a.ctas > 1 ? 3 : 2);    // both streams; in a cluster sums are kept in place 0
            mbar_init(&sh.s_full[lane], 1);
            mbar_init(&sh.p_full[lane], 8);
            mbar_init(&sh.o_full[lane], 1);
            mbar_init(&sh.drained[lane], 1);
            mbar_init(&sh.job_full[lane], 1);
            mbar_init(&sh.job_empty[lane], 3 + 16 + (Q8 ? kConvert : 0));        // a warp each: loads, products, softmax, conversion
        }
        if (lane == 2) {
            mbar_init(&sh.ready, 1);
            mbar_init(&sh.taken, a.ctas);
            sh.tensor = 0;
        }
        mbar_fence_init();
        if (lane == 3) {
            tma_prefetch_desc(&q_map);
            tma_prefetch_desc(&k_map);
            tma_prefetch_desc(&v_map);
        }
    } else if (warp == 3) {
        tmem_alloc(&sh.tmem, 512);
        tmem_relinquish();
    }
    pdl_wait();                                             // what follows reads what earlier kernels wrote
    pdl_launch_dependents();
    if (warp == 2) more = plan.start(a, lane, blockIdx.x / a.ctas, gridDim.x / a.ctas);     // the same for the whole cluster
    tc_fence_before();
    __syncwarp();
    if (a.ctas > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // this CTA's barriers are set up
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;                          // S0, S1 at 0, 128; O0, O1 at 256, 256 + D; of heads of 64 P0, P1 at 384, 448
    bool cluster_up = a.ctas == 1;                          // the neighbours' barriers are, as far as this warp knows
    auto cluster_wait = [&] {
        if (!cluster_up) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        cluster_up = true;
    };

    // Segment number `i` of this CTA, when warp 2 has worked it out; false = a wait ran out.  For whole warps.
    auto job_of = [&](int i) { return __all_sync(0xFFFFFFFFu, mbar_wait(&sh.job_full[i & 1], (i >> 1) & 1, wl)); };
    // The calling warp is done with it.
    auto job_done = [&](int i) {
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.job_empty[i & 1]);
    };

    if (warp < 4) {
        set_registers<false, Q8 ? 56 : 64>();
        if (warp == 0) {
            // ---- tiles of keys and values: 16-bit ones straight into the stages, 8-bit ones into the raw ring
            constexpr int kRing = Q8 ? Geo::kRaw : kStages;
            constexpr int kBytes = Q8 ? Geo::kRawBytes : kTileBytes;
            constexpr int kParts = Q8 ? 1 : kSlabs;              // copies per page
            uint8_t *ring = Q8 ? raws : stages;
            uint64_t *full = Q8 ? sh.raw_full : sh.full, *empty = Q8 ? sh.raw_empty : sh.empty;
            const int per = kTile >> a.kv.page_shift;            // pages per tile
            const int pg = lane / kParts, part = lane % kParts;
            const int beyond = (int)min((long long)a.kv.layers * a.kv.num_pages * a.kv.heads << a.kv.page_shift, 2147483647LL);
            int issued = 0;
            bool ok = true;
            for (int i = 0; ok; ++i) {
                if (!job_of(i)) { ok = false; break; }
                const Job &w = sh.job[i & 1];
                if (!w.more) break;
                const int total = w.c.total, head = w.seg.head;
                const int32_t *table = a.kv.table + (long long)w.seg.b * a.kv.width;
                // page of this lane's copy of this CTA's tile j, as a row of the maps (out of range: zeros are loaded)
                auto row_of = [&](int j) {
                    const int p = w.tile(j) * kTile + (pg << a.kv.page_shift);
                    int page = -1;
                    if (j < w.nt && pg < per && p < total && debug_check(p >= 0 && (p >> a.kv.page_shift) < a.kv.width, a.kv.status, 71)) page = __ldg(table + (p >> a.kv.page_shift));
                    if (page < 0 || page >= a.kv.num_pages) return beyond;
                    return (int)kv_row(a.kv, a.kv.layer, page, head, 0);
                };
                auto load = [&](bool is_v, int row) {
                    const int s = issued % kRing;
                    if (!debug_check(row >= 0 && row <= beyond && (row == beyond || (row & ((1 << a.kv.page_shift) - 1)) == 0), a.kv.status, 72)) row = beyond;
                    if (issued >= kRing && !mbar_wait(&empty[s], ((issued / kRing) - 1) & 1, wl)) ok = false;
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) return;
                    if (lane == 0) mbar_arrive_expect_tx(&full[s], (uint32_t)(kBytes + (Q8 ? kTile : 0)));
                    __syncwarp();
                    if (pg < per && !(a.lose_stage > 0 && blockIdx.x == 0 && issued == a.lose_stage - 1)) {
                        uint8_t *dst = ring + (size_t)s * kBytes + part * kSlabBytes + ((size_t)pg << a.kv.page_shift) * (Q8 ? D : 128);
                        tma_load_2d(dst, is_v ? &v_map : &k_map, part * 64, row, &full[s]);
                        // the page's exponents; zeros have any
                        if constexpr (Q8)
                            bulk_load(sh.exps[s] + (pg << a.kv.page_shift), (is_v ? a.kv.v_exps : a.kv.k_exps) + (row < beyond ? row : 0),
                                      1u << a.kv.page_shift, &full[s]);
                    }
                    ++issued;
                };
                const int ahead = w.one ? 2 : 1, nt = w.nt;
                int r0 = row_of(0), r1 = row_of(1);          // of value tiles j, j + 1
#pragma unroll 1
                for (int x = 0; x < min(ahead, nt) && ok; ++x) load(false, x ? r1 : r0);
#pragma unroll 1
                for (int j = 0; j < nt && ok; ++j) {
                    const int r2 = row_of(j + 2);
                    load(true, r0);
                    if (ok && j + ahead < nt) load(false, ahead == 2 ? r2 : r1);
                    r0 = r1;
                    r1 = r2;
                }
                job_done(i);
            }
            if (!ok && lane == 0) report_timeout(a.kv.status);
            // no copy may be in flight when the CTA ends
            for (int x = max(0, issued - kRing); x < issued; ++x)
                if (!mbar_wait(&full[x % kRing], (x / kRing) & 1, wl) && lane == 0) report_timeout(a.kv.status);
        } else if (warp != 2) {
            // ---- products of stream st.  The whole warp walks through the loop and one lane issues: what the instructions take
            // must be known to be the same for all lanes (hence the shuffles), or every operand is moved to the uniform registers
            // by itself, at 100 cycles and more an instruction against the 64 that it runs.
            constexpr uint32_t kFmt = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
            constexpr uint32_t kCommon = (1u << 4) | (kFmt << 7) | (kFmt << 10) | ((uint32_t)(kTile >> 4) << 24);
            constexpr uint32_t kIdescS = kCommon | ((uint32_t)(kTile >> 3) << 17);
            constexpr uint32_t kIdescO = kCommon | ((uint32_t)(D >> 3) << 17) | (1u << 16);       // second operand MN-major
            auto uniform = [](int x) { return __shfl_sync(0xFFFFFFFFu, x, 0); };
            const int st = uniform(warp == 3);
            const uint32_t t0 = uniform(tmem), s_at = t0 + st * kTile, o_at = t0 + 256 + st * D;
            const uint32_t p_at = kOwnP ? t0 + kPAt + st * (kTile / 2) : s_at + (Q8 ? 32 : 0);
            const uint64_t q_desc = make_desc(smem_u32(q_s)), k_desc = make_desc(smem_u32(stages)), v_desc = make_desc_mn(smem_u32(stages));
            uint64_t *q_full = sh.q_full, *q_empty = sh.q_empty;
            const bool issuer = elect_one();
            int base = 0, at = 0;                            // tiles of earlier segments; tiles gone through
            int steps = 0, uses0 = 0, uses1 = 0;
            bool ok = true;
            for (int i = 0; ok; ++i) {
                if (!job_of(i)) { ok = false; break; }
                const Job &w = sh.job[i & 1];
                if (!uniform(w.more)) break;
                const bool one = uniform(w.one) != 0;
                const int nt = uniform(w.nt), n = uniform(w.n[st]);
                auto wait = [&](uint64_t *bar, int parity) {
                    ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity & 1, wl));
                    tc_fence_after();
                    return ok;
                };
                auto k_place = [&](int j) { return one ? (j < 2 ? j : 2 * j - 1) : 2 * j; };
                auto v_place = [&](int j) { return one ? (j == nt - 1 ? 2 * nt - 1 : 2 + 2 * j) : 2 * j + 1; };
                // Tile x of the line.  Both streams go through ALL tiles in order and both free each of them, the other stream's
                // too: a barrier's parity tells two neighbouring rounds of the ring apart and no more, so neither stream may
                // get a round ahead of a tile that the other one has not seen arrive.
                auto reach = [&](int x) {
                    for (; at < x; ++at) {
                        if (!wait(&sh.full[at % kStages], at / kStages)) return false;
                        if (lane == 0) mbar_arrive(&sh.empty[at % kStages]);
                    }
                    ++at;
                    return wait(&sh.full[x % kStages], x / kStages);
                };
                // A stream's products are issued in one go: side by side, both streams would wait for the tensor cores and
                // then for the exponentials together, instead of in turn.
                auto lock = [&] {
                    bool got = true;
                    if (lane == 0) {
                        const long long t = clock64();
                        while (got && atomicExch(&sh.tensor, 1u) != 0) got = clock64() - t < wl;
                    }
                    ok = __all_sync(0xFFFFFFFFu, got);
                    return ok;
                };
                auto unlock = [&] {
                    __syncwarp();
                    if (lane == 0) atomicExch(&sh.tensor, 0u);
                };
                auto issue_scores = [&](int j, int s) {
                    const uint64_t qd = q_desc + (one ? 0 : st * (kTileBytes >> 4)), kd = k_desc + s * (kTileBytes >> 4);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        umma_f16(s_at, qd + ((k >> 2) * (kSlabBytes >> 4) + 2 * (k & 3)), kd + ((k >> 2) * (kSlabBytes >> 4) + 2 * (k & 3)),
                                 kIdescS, k != 0);
                    tc_commit(&sh.s_full[st]);
                    tc_commit(&sh.empty[s]);
                    if (j == n - 1) {
                        tc_commit(&q_empty[0]);
                        if (!one) tc_commit(&q_empty[1]);
                    }
                };
                // the queries: both streams wait for and free all row tiles, for the same reason
                wait(&q_full[0], uses0++);
                if (ok && !one) wait(&q_full[1], uses1++);
                if (ok && n > 0) {
                    const int x = base + k_place(one ? st : 0);
                    if (reach(x) && lock()) {
                        if (issuer) issue_scores(0, x % kStages);
                        unlock();
                    }
                } else if (ok && issuer) {
                    tc_commit(&q_empty[0]);                  // a cluster with fewer tiles than streams
                }
#pragma unroll 1
                for (int j = 0; j < n && ok; ++j) {
                    const int vj = one ? 2 * j + st : j, x = base + v_place(vj), s = x % kStages;
                    const bool more = j + 1 < n;
                    const int y = more ? base + k_place(one ? vj + 2 : j + 1) : 0;
                    if (!reach(x) || (more && !reach(y))) break;
                    // The turn is taken before the weights are there, to have its cost behind us -- but not for a segment's first tile,
                    // whose weights may wait for the other stream's last products of the segment before.
                    if (j == 0 ? !wait(&sh.p_full[st], steps) || !lock() : !lock()) break;
                    if (j > 0 && !wait(&sh.p_full[st], steps)) {
                        unlock();
                        break;
                    }
                    ++steps;
                    const uint64_t vd = v_desc + s * (kTileBytes >> 4);
                    if (issuer) {
                        if (j == 0) umma_f16_ta(o_at, p_at, vd, kIdescO, 0);
                        else umma_f16_ta(o_at, p_at, vd, kIdescO, 1);
#pragma unroll
                        for (int k = 1; k < kTile / 16; ++k) umma_f16_ta(o_at, p_at + 8 * k + (Q8 && !kOwnP && k >= kTile / 32 ? 32 : 0), vd + 128 * k, kIdescO, 1);
                        tc_commit(&sh.empty[s]);
                        // At d = 128 the next scores go to the columns that hold the weights of the product just issued, with no wait
                        // between: this relies on the tensor core running the products of a CTA in the order in which one thread
                        // issues them, also where their sums lie in different columns.  (A wait there changes no bit of any result and
                        // costs 6 % of a long prompt and 10 % of 1024 rows at 6000.)  What else reads or writes these columns, or O, is
                        // behind the commit of the next scores, which counts all products issued before it.
                        if (more) issue_scores(j + 1, y % kStages);
                        else tc_commit(&sh.o_full[st]);
                    }
                    unlock();
                }
                base += 2 * nt;
                if (ok && at < base) {                       // the other stream's last tiles
                    reach(base - 1);
                    if (ok && lane == 0) mbar_arrive(&sh.empty[(base - 1) % kStages]);
                }
                job_done(i);
            }
            // no product may be running when the CTA ends, nor when TMEM is given back
            if (issuer) tc_commit(&sh.drained[st]);
            if (!mbar_wait(&sh.drained[st], 0, wl)) ok = false;
            if (!ok && lane == 0) report_timeout(a.kv.status);
        } else {
            // ---- the plan, and queries
            if (lane == 0) {
                const int tokens = ManyRows::per_tile(a);
                const uint32_t bytes = (uint32_t)(tokens * a.group * 128 * kSlabs);
                int uses0 = 0, uses1 = 0;
                bool ok = true;
#pragma unroll 1
                for (int i = 0; ok; ++i) {
                    if (i >= 2 && !mbar_wait(&sh.job_empty[i & 1], ((i >> 1) - 1) & 1, wl)) { ok = false; break; }
                    Job &w = sh.job[i & 1];
                    if (more) more = plan.next(a, w.seg);
                    w.more = 0;
                    if (more) {
                        w.c = plan.c;
                        w.set(a, rank);
                    }
                    mbar_arrive(&sh.job_full[i & 1]);
                    if (!more) break;
                    const int tiles = w.one ? 1 : 2, y = w.seg.head * a.group;
                    int z = plan.c.row0 + w.seg.rt * (int)a.by_rows.d;
                    if (!debug_check(z >= 0 && z < a.kv.rows && w.seg.head < a.kv.heads, a.kv.status, 73)) z = 0;
#pragma unroll 1
                    for (int st = 0; st < tiles && ok; ++st) {
                        int &uses = st ? uses1 : uses0;
                        if (uses > 0) ok = mbar_wait(&sh.q_empty[st], (uses - 1) & 1, wl);
                        if (!ok) break;
                        mbar_arrive_expect_tx(&sh.q_full[st], bytes);
#pragma unroll
                        for (int p = 0; p < kSlabs; ++p)
                            tma_load_3d(q_s + st * kTileBytes + p * kSlabBytes, &q_map, p * 64, y, z + st * tokens, &sh.q_full[st]);
                        ++uses;
                    }
                }
                if (!ok) report_timeout(a.kv.status);
                // no copy may be in flight when the CTA ends
                if (uses0 > 0 && !mbar_wait(&sh.q_full[0], (uses0 - 1) & 1, wl)) report_timeout(a.kv.status);
                if (uses1 > 0 && !mbar_wait(&sh.q_full[1], (uses1 - 1) & 1, wl)) report_timeout(a.kv.status);
            }
        }
    } else if (warp < 20) {
        set_registers<true, Q8 ? 96 : 104>();
        // ---- softmax of stream st; a thread has positions 64 half .. of a tile of its row
        const int st = warp >= 12 ? 1 : 0, half = (warp >> 2) & 1 ? 0 : 1;      // warps 4-7, 12-15: the first half
        const int row = tid & 127;                           // TMEM lane
        const int pair_bar = 4 + 4 * st + (warp & 3);        // barrier of the two warps that have the same rows
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;    // (warp % 4) x 32 lanes, in the address's upper half
        const uint32_t ts = tmem + lanes + st * kTile + 64 * half, to = tmem + lanes + 256 + st * D;
        const uint32_t tp = kOwnP ? tmem + lanes + kPAt + st * (kTile / 2) + 32 * half : Q8 ? ts + 32 : tmem + lanes + st * kTile + 32 * half;
        const int row_tok = a.by_group.div(row);
        int steps = 0, items0 = 0, items1 = 0, joins = 0, base = 0;
        bool dead = false;
        for (int i = 0;; ++i) {
            if (bar_or(1, 512, dead || !job_of(i))) {        // all softmax warps go on, or none (they meet at barriers)
                report_timeout(a.kv.status);
                break;
            }
            const Job &w = sh.job[i & 1];
            if (!w.more) break;
            const Chunk &c = w.c;
            const Segment &seg = w.seg;
            const int n_mine = w.n[st];
            const int first_tok = seg.rt * (int)a.by_rows.d + (w.one ? 0 : st * ManyRows::per_tile(a));
            const int tok = first_tok + row_tok;              // of this row; may lie behind the chunk
            // A row of the result.  The others hold the queries of other tokens, or (behind 128 / group x group) whatever was in shared
            // memory: they take part in nothing.
            const bool valid = row < ManyRows::per_tile(a) * a.group && tok < c.len;
            const int limit = a.mask ? c.total : c.upto(min(tok, c.len - 1));
            const int all_seen = a.mask ? c.ctx : c.upto(min(first_tok, c.len - 1));    // by every row
            float m = -INFINITY, l = 0.f;                     // m in powers of two
            const float scale = a.scale_log2;
#pragma unroll 1
            for (int j = 0; j < n_mine; ++j) {
                const int vj = w.one ? 2 * j + st : j, p0 = w.tile(vj) * kTile, v_at = base + w.v_place(vj);
                if (!dead && !mbar_wait(&sh.s_full[st], steps & 1, wl)) {
                    report_timeout(a.kv.status);
                    dead = true;
                }
                const bool ragged = !Q8 && vj == w.nt - 1 && p0 + kTile > c.total;
                if (ragged)                                   // the values: their places behind the end are cleared
                    if (!dead && !mbar_wait(&sh.full[v_at % kStages], (v_at / kStages) & 1, wl)) {
                        report_timeout(a.kv.status);
                        dead = true;
                    }
                dead = __any_sync(0xFFFFFFFFu, dead);
                ++steps;
                tc_fence_after();
                // With a 16-bit cache a thread holds its 64 scores, and weights (where they have no columns of their own) go to the first
                // half of the tile's columns.  With an 8-bit cache there are fewer registers (the converting warps have the rest): 32
                // scores at a time, the first 32 read twice, weights to the place of the second 32.  1024 rows x 4 heads of 128 at 6000 positions, 8 bits,
                // 167 us so and 170 with 64 held (fp16 145 and 157; 148 items of 244 rows, heads of 64, 124 and 123); the 16-bit
                // kernel, heads of 64, 124 so and 118 with 64 held.
                float s[64];
                uint32_t *su = reinterpret_cast<uint32_t *>(s);
                const bool masked = p0 + kTile > all_seen;
                tmem_ld32(ts, su);
                if constexpr (!Q8) tmem_ld32(ts + 32, su + 32);
                // What a row sees of 32 positions, and the largest score.
                auto seen = [&](int p) {
                    const int n = min(max(limit - p, 0), 32);
                    uint32_t see = n == 32 ? 0xFFFFFFFFu : (1u << n) - 1u;
                    if (a.mask && p + 32 > c.ctx && debug_check(c.row0 + min(tok, c.len - 1) < a.kv.rows && p - c.ctx > -32, a.kv.status, 74)) {
                        const uint32_t *mask = a.mask + (long long)(c.row0 + min(tok, c.len - 1)) * a.mask_words;
                        const int j0 = p - c.ctx;             // place in the chunk of bit 0; context below 0
                        const int w0 = j0 >> 5;               // floor; -1 at the least
                        const uint32_t lo = w0 < 0 ? 0xFFFFFFFFu : w0 < a.mask_words ? mask[w0] : 0u;
                        const uint32_t hi = w0 + 1 < a.mask_words ? mask[w0 + 1] : 0u;
                        see &= __funnelshift_r(lo, hi, j0 & 31);
                    }
                    return see;
                };
                auto hide = [&](float *x, uint32_t see) {
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (!(see >> k & 1)) x[k] = -INFINITY;
                };
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                auto largest = [&](const float *x, int n) {
#pragma unroll
                    for (int k = 0; k < n; k += 8)
#pragma unroll
                        for (int y = 0; y < 4; ++y) mx[y] = fmaxf(fmaxf(mx[y], x[k + 2 * y]), x[k + 2 * y + 1]);
                };
                uint32_t see = 0xFFFFFFFFu;                   // of the first 32
                tmem_ld_wait_for(su);
                if constexpr (Q8) tmem_ld32(ts + 32, su + 32);
                else tmem_ld_wait_for(su + 32);
                if (masked) hide(s, see = seen(p0 + 64 * half));
                if constexpr (Q8) {
                    largest(s, 32);
                    tmem_ld_wait_for(su + 32);
                }
                if (masked) hide(s + 32, seen(p0 + 64 * half + 32));
                if constexpr (Q8) largest(s + 32, 32);
                else largest(s, 64);
                const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale;
                const bool over = valid && top - m > kSlack;  // -inf - -inf is NaN: no
                tc_fence_before();
                // Both halves of a row have one maximum; both have been read, weights may take their place.  The two warps that have
                // these 32 rows meet, nobody else has to.
                const bool raise = bar_or(pair_bar, 64, over);
                tc_fence_after();
                if (raise) {
                    float *pass = &sh.l[st][row];
                    if (half) *pass = top;
                    bar_sync(pair_bar, 64);
                    float mn;
                    if (!half) *pass = mn = fmaxf(fmaxf(m, top), *pass);
                    bar_sync(pair_bar, 64);
                    if (half) mn = *pass;
                    const float f = mn > -INFINITY ? ex2(m - mn) : 1.f;
                    l *= f;
                    m = mn;
                    if (j > 0) {
#pragma unroll 1
                        for (int k = half * (D / 2); k < half * (D / 2) + D / 2; k += 16) {
                            uint32_t r[16];
                            tmem_ld16(to + k, r);
                            tmem_ld_wait16(r);
#pragma unroll
                            for (int x = 0; x < 16; ++x) r[x] = __float_as_uint(__uint_as_float(r[x]) * f);
                            tmem_st16(to + k, r);
                        }
                        tmem_st_wait();
                    }
                    tc_fence_before();
                    bar_sync(pair_bar, 64);                   // the second product begins when one half has its weights
                    tc_fence_after();
                }
                const float off = (m > -INFINITY ? m : 0.f) - Lift<T>::value;
                const uint64_t scale2 = pair(scale, scale), off2 = pair(-off, -off);
                uint64_t sum0 = 0, sum1 = 0;
                // weights of some scores, packed and stored at column c0
                constexpr int kAtOnce = Q8 ? 16 : 32;
                auto weights = [&](const float *of, int c0) {
                    uint32_t p[kAtOnce / 2];
#pragma unroll
                    for (int k = 0; k < kAtOnce; k += 2) {
                        uint64_t x = fma2(pair(of[k], of[k + 1]), scale2, off2);
                        float lo, hi;
                        unpair(x, lo, hi);
                        lo = ex2(lo);
                        hi = ex2(hi);
                        x = pair(lo, hi);
                        if (k & 2) sum1 = add2(sum1, x);
                        else sum0 = add2(sum0, x);
                        p[k / 2] = pack2<T>(lo, hi);
                    }
                    if constexpr (Q8) tmem_st8(tp + c0, p);
                    else tmem_st16(tp + c0, p);
                };
                if constexpr (Q8) {
                    tmem_ld16(ts, su);
                    weights(s + 32, 16);
                    tmem_ld16(ts + 16, su + 16);
                    weights(s + 48, 24);
                    tmem_ld_wait16(su);
                    tmem_ld_wait16(su + 16);
                    if (masked) hide(s, see);
                    weights(s, 0);
                    weights(s + 16, 8);
                } else {
                    weights(s, 0);
                    weights(s + 32, 16);
                }
                float a0, a1;
                unpair(add2(sum0, sum1), a0, a1);
                l += a0 + a1;
                if (ragged) {                                 // the places behind the end among this half's positions
                    const int end = min(max(c.total - p0, 64 * half), 64 * half + 64), rows = 64 * half + 64 - end;
                    uint8_t *tile = stages + (size_t)(v_at % kStages) * kTileBytes + end * 128;
#pragma unroll 1
                    for (int y = row; y < rows * 8; y += kTile)
#pragma unroll
                        for (int p = 0; p < kSlabs; ++p) *reinterpret_cast<uint4 *>(tile + p * kSlabBytes + y * 16) = make_uint4(0, 0, 0, 0);
                    fence_async_smem();
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.p_full[st]);
            }
            // ---- the segment's result
            base += 2 * w.nt;
            const int heads = a.kv.heads * a.group;
            if (half) sh.l[st][row] = l;
            bar_sync(2 + st, 256);
            if (!half) {
                sh.l[st][row] += l;
                sh.m[st][row] = m;
            }
            if (w.n[0] > 0) {
                if ((w.one || st == 0) && !dead && !mbar_wait(&sh.o_full[0], items0 & 1, wl)) {
                    report_timeout(a.kv.status);
                    dead = true;
                }
                ++items0;
            }
            if (w.n[1] > 0) {
                if ((w.one || st == 1) && !dead && !mbar_wait(&sh.o_full[1], items1 & 1, wl)) {
                    report_timeout(a.kv.status);
                    dead = true;
                }
                ++items1;
            }
            dead = __any_sync(0xFFFFFFFFu, dead);
            bar_sync(1, 512);
            tc_fence_after();
            // A thread has a row and some OCTETS of its elements, o0, o0 + o_step, ...: with two row tiles its stream's row and
            // half of the octets; with one, a quarter of the octets from both streams, or in a cluster its CTA's share of them.
            const bool joined = a.ctas > 1;
            const int prow = w.one ? row : st * kTile + row, quarter = 2 * st + half;
            const int d0 = w.one ? quarter * (D / 4) : half * (D / 2), d1 = w.one ? d0 + D / 4 : d0 + D / 2;
            const int o0 = joined ? quarter * a.ctas + rank : d0 / 8;      // in a cluster octet o is with CTA o % ctas
            const int o_step = joined ? 4 * a.ctas : 1, o_end = joined ? D / 8 : d1 / 8;
            float f0 = 1.f, f1 = 0.f;
            l = sh.l[w.one ? 0 : st][row];
            if (w.one) {
                const float ma = sh.m[0][row], mb = sh.m[1][row];
                m = fmaxf(ma, mb);
                f0 = m > -INFINITY ? ex2(ma - m) : 0.f;
                f1 = m > -INFINITY ? ex2(mb - m) : 0.f;
                l = f0 * l + f1 * sh.l[1][row];
            }
            const bool split = seg.c0 != seg.c1;
            const long long at = (long long)(c.row0 + tok) * heads + seg.head * a.group + row - row_tok * a.group;
            const bool own = (w.tile(max(w.nt - 1, 0)) + 1) * kTile > c.ctx;      // the chunk's own tokens are among the positions
            float *part = a.part + ((size_t)blockIdx.x * 2 + seg.slot) * part_floats(D);
            float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;       // a NaN sum stays one
            auto put = [&](int o, const float *x) {            // an octet of the result
                if (valid && debug_check(at >= 0 && at < (long long)a.kv.rows * heads && o < D / 8, a.kv.status, 75))
                    reinterpret_cast<uint4 *>(static_cast<T *>(a.out) + at * D)[o] =
                        make_uint4(pack2<T>(x[0] * inv, x[1] * inv), pack2<T>(x[2] * inv, x[3] * inv), pack2<T>(x[4] * inv, x[5] * inv),
                                   pack2<T>(x[6] * inv, x[7] * inv));
            };
            auto put_part = [&](int o, const float *x) {
                if (!valid || !debug_check((unsigned)seg.slot < 2 && o < D / 8, a.kv.status, 76)) return;
                float4 *dst = reinterpret_cast<float4 *>(part) + (size_t)(2 * o) * kPartRows + prow;
                __stcg(dst, make_float4(x[0], x[1], x[2], x[3]));
                __stcg(dst + kPartRows, make_float4(x[4], x[5], x[6], x[7]));
            };
            const int per = D / 8 / a.ctas;                    // octets of a CTA of a cluster
            if (joined) {
                cluster_wait();
                if (tid == 128) mbar_arrive_expect_tx(&sh.ready, (uint32_t)(kTile * ((a.ctas - 1) * per * 32 + a.ctas * 8)));
                // what was sent the last time has been read
                if (joins > 0 && !dead && !mbar_wait_cluster(&sh.taken, (joins - 1) & 1, wl)) {
                    report_timeout(a.kv.status);
                    dead = true;
                }
                if (quarter == 0)
                    for (int x = 0; x < a.ctas; ++x) st_async(&sent_ml[rank * kTile + row], make_float2(m, l), &sh.ready, x);
            }
            // sums of this CTA: 16 elements at a time from TMEM to the result, the part, or the octet's CTA
            auto take = [&](int of, uint32_t addr, int d, float *x) {         // sums of stream `of`
                uint32_t r[16];
                tmem_ld16(addr, r);
                tmem_ld_wait16(r);
                float odd = 0.f;
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    x[k] = __uint_as_float(r[k]);
                    odd = fmaf(x[k], 0.f, odd);
                }
                if constexpr (!Q8) {
                    if (own && valid && odd != 0.f) {          // NaN
                        float y[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k) y[k] = x[k];
                        repair<T, D>(a, w, of, row, tok, sh.m[of][row], d, y);
#pragma unroll
                        for (int k = 0; k < 16; ++k) x[k] = y[k];
                    }
                }
            };
#pragma unroll 1
            for (int d = d0; d < d1; d += 16) {
                float x[16];
                if (w.n[w.one ? 0 : st] > 0) {
                    take(w.one ? 0 : st, w.one ? tmem + lanes + 256 + d : to + d, d, x);
                } else {
#pragma unroll
                    for (int k = 0; k < 16; ++k) x[k] = 0.f;
                }
                if (w.one) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) x[k] = f0 > 0.f || f0 != f0 ? f0 * x[k] : 0.f;
                    if (w.n[1] > 0) {
                        float z[16];
                        take(1, tmem + lanes + 256 + D + d, d, z);
#pragma unroll
                        for (int k = 0; k < 16; ++k) x[k] += f1 > 0.f || f1 != f1 ? f1 * z[k] : 0.f;
                    }
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (joined) {
                        const int o = d / 8 + k, to = o & (a.ctas - 1), n = o / a.ctas;
                        const float4 y = make_float4(x[8 * k], x[8 * k + 1], x[8 * k + 2], x[8 * k + 3]);
                        const float4 z = make_float4(x[8 * k + 4], x[8 * k + 5], x[8 * k + 6], x[8 * k + 7]);
                        if (to == rank) {
                            kept[2 * n * kTile + row] = y;
                            kept[(2 * n + 1) * kTile + row] = z;
                        } else {                               // its place there: 0 for the next CTA in the ring
                            const int place = (((rank - to - 1) & (a.ctas - 1)) * per + n) * 2 * kTile + row;
                            if (!debug_check(place >= 0 && place + kTile < kTile * D / 4 / kMaxCtas * (kMaxCtas - 1), a.kv.status, 79)) continue;
                            float4 *at = sent + place;
                            st_async(at, y, &sh.ready, to);
                            st_async(at + kTile, z, &sh.ready, to);
                        }
                    } else if (split) {
                        put_part(d / 8 + k, x + 8 * k);
                    } else {
                        put(d / 8 + k, x + 8 * k);
                    }
                }
            }
            if (joined) {
                if (!dead && !mbar_wait_cluster(&sh.ready, joins & 1, wl)) {
                    report_timeout(a.kv.status);
                    dead = true;
                }
                bar_sync(1, 512);                             // what is kept is in place
                m = -INFINITY;
                for (int x = 0; x < a.ctas; ++x) m = fmaxf(m, sent_ml[x * kTile + row].x);
                l = 0.f;
                for (int x = 0; x < a.ctas; ++x) {
                    const float2 p = sent_ml[x * kTile + row];
                    l += m > -INFINITY ? ex2(p.x - m) * p.y : 0.f;
                }
                inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
#pragma unroll 1
                for (int o = o0; o < o_end; o += o_step) {
                    float x8[8] = {};
                    for (int x = 0; x < a.ctas; ++x) {
                        const float f = m > -INFINITY ? ex2(sent_ml[x * kTile + row].x - m) : 0.f;
                        const float4 *at = (x == rank ? kept : sent + ((x - rank - 1) & (a.ctas - 1)) * per * 2 * kTile) + o / a.ctas * 2 * kTile + row;
                        const float4 y = at[0], z = at[kTile];
                        if (f > 0.f || f != f) {
                            x8[0] += f * y.x, x8[1] += f * y.y, x8[2] += f * y.z, x8[3] += f * y.w;
                            x8[4] += f * z.x, x8[5] += f * z.y, x8[6] += f * z.z, x8[7] += f * z.w;
                        }
                    }
                    if (split) put_part(o, x8);
                    else put(o, x8);
                }
                fence_async_smem();                           // the next queries come to the same place
                bar_sync(1, 512);
                if (tid - 128 < a.ctas) mbar_arrive_cluster(mapa_rank(smem_u32(&sh.taken), tid - 128));
                if (tid == 128) mbar_arrive(&sh.q_empty[0]);
                dead = __any_sync(0xFFFFFFFFu, dead);
                ++joins;
            }
            bool done = !split;
            if (split) {
                if (joined ? quarter == 0 : w.one ? quarter == 0 : half == 0) {
                    __stcg(part + kPartRows * D + prow, m);
                    __stcg(part + kPartRows * (D + 1) + prow, l);
                }
                __threadfence();
                bar_sync(1, 512);
                // CTAs of the same rank join the same octets
                if (tid == 128 && debug_check(seg.c0 >= 0 && (seg.c1 + 1) * a.ctas <= (int)gridDim.x, a.kv.status, 77))
                    sh.ticket = atomicAdd(a.tickets + seg.c0 * a.ctas + rank, 1u);
                bar_sync(1, 512);
                done = *reinterpret_cast<volatile unsigned *>(&sh.ticket) == (unsigned)(seg.c1 - seg.c0);
                if (done) {                                       // the last of the item's workers: join the parts in order
                    __threadfence();
                    if (tid == 128) a.tickets[seg.c0 * a.ctas + rank] = 0;
                    auto part_of = [&](int i) {
                        return a.part + ((size_t)(i * a.ctas + rank) * 2 + (i == seg.c0 ? seg.slot0 : 0)) * part_floats(D);
                    };
                    m = -INFINITY;
#pragma unroll 4
                    for (int i = seg.c0; i <= seg.c1; ++i) m = fmaxf(m, __ldcg(part_of(i) + kPartRows * D + prow));
                    l = 0.f;
#pragma unroll 4
                    for (int i = seg.c0; i <= seg.c1; ++i) {
                        const float *ps = part_of(i);
                        const float f = m > -INFINITY ? ex2(__ldcg(ps + kPartRows * D + prow) - m) : 0.f;
                        l += f * __ldcg(ps + kPartRows * (D + 1) + prow);
                    }
                    inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
#pragma unroll 1
                    for (int o = o0; o < o_end; o += 2 * o_step) {           // two octets at a time
                        float x[16] = {};
#pragma unroll 2
                        for (int i = seg.c0; i <= seg.c1; ++i) {
                            const float *ps = part_of(i);
                            const float f = m > -INFINITY ? ex2(__ldcg(ps + kPartRows * D + prow) - m) : 0.f;
                            float4 y[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const int oo = o + (k >> 1) * o_step;
                                y[k] = valid && oo < o_end ? __ldcg(reinterpret_cast<const float4 *>(ps) + (size_t)(2 * oo + (k & 1)) * kPartRows + prow)
                                                           : make_float4(0.f, 0.f, 0.f, 0.f);
                            }
                            if (f > 0.f || f != f) {
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    x[4 * k] += f * y[k].x;
                                    x[4 * k + 1] += f * y[k].y;
                                    x[4 * k + 2] += f * y[k].z;
                                    x[4 * k + 3] += f * y[k].w;
                                }
                            }
                        }
#pragma unroll
                        for (int k = 0; k < 2; ++k)
                            if (o + k * o_step < o_end) put(o + k * o_step, x + 8 * k);
                    }
                }
            }
            if (done && valid && a.lse && o0 == 0) a.lse[at] = (m > -INFINITY ? m - Lift<T>::value + log2f(l) : -INFINITY) * 0.69314718055994531f;
            tc_fence_before();
            bar_sync(1, 512);                                // all have read O, sh.m and sh.l
            job_done(i);
        }
    } else {
        // ---- 8-bit tiles -> 16-bit tiles
        if constexpr (Q8) {
            set_registers<false, 32>();
            constexpr int kPieces = D / 16;                  // 16-byte pieces of a position
            const int t = tid - 640;
            int done = 0;                                    // tiles
            bool ok = true;
            for (int i = 0; ok; ++i) {
                if (!job_of(i)) { ok = false; break; }
                const Job &w = sh.job[i & 1];
                if (!w.more) break;
                const Chunk c = w.c;
#pragma unroll 1
                for (int x = 0, kj = 0, vj = 0; x < 2 * w.nt && ok; ++x, ++done) {
                    const bool is_v = x == w.v_place(vj);
                    const int p0 = w.tile(is_v ? vj++ : kj++) * kTile;
                    const int rs = done % Geo::kRaw, s = done % kStages;
                    bool got = mbar_wait(&sh.raw_full[rs], (done / Geo::kRaw) & 1, wl);
                    if (done >= kStages) got = got && mbar_wait(&sh.empty[s], ((done / kStages) - 1) & 1, wl);
                    ok = __all_sync(0xFFFFFFFFu, got);
                    if (!ok) break;
                    const uint8_t *raw = raws + (size_t)rs * Geo::kRawBytes;
                    uint8_t *tile = stages + (size_t)s * kTileBytes;
                    // A thread has piece `piece` of every (32 x kConvert / kPieces)-th position, two at a time (four spill): both
                    // loads before the first store, which the compiler would not move a load across.  Pieces of the second slab go by the neighbouring
                    // position, whose swizzle spreads the slabs over the banks.
                    constexpr int kMine = kTile * kPieces / (32 * kConvert);
                    const int piece = t % kPieces, pos0 = (t / kPieces) ^ (piece >> 2 & 1);
                    uint8_t *dst = tile + (piece >> 2) * kSlabBytes + pos0 * 128;
                    const int ch = ((piece & 3) * 2 ^ (pos0 & 7)) << 4;      // two chunks of the slab's 128-byte row, swizzled by the row
#pragma unroll 1
                    for (int n0 = 0; n0 < kMine; n0 += 2) {
                        uint4 codes[2];
                        int exps[2];
#pragma unroll
                        for (int n = 0; n < 2; ++n) {
                            const int pos = pos0 + (n0 + n) * (kTile / kMine);
                            codes[n] = *reinterpret_cast<const uint4 *>(raw + pos * D + piece * 16);
                            exps[n] = sh.exps[rs][pos];
                        }
                        if (p0 + kTile > c.ctx) {                  // unused places and the code of NaN count as 0
#pragma unroll
                            for (int n = 0; n < 2; ++n) {
                                const bool use = p0 + pos0 + (n0 + n) * (kTile / kMine) < c.total;
                                auto plain = [&](uint32_t u) { return use ? u & ~__vcmpeq4(u & 0x7F7F7F7Fu, 0x7F7F7F7Fu) : 0u; };
                                codes[n] = make_uint4(plain(codes[n].x), plain(codes[n].y), plain(codes[n].z), plain(codes[n].w));
                            }
                        }
#pragma unroll
                        for (int n = 0; n < 2; ++n) {
                            const uint32_t u[4] = {codes[n].x, codes[n].y, codes[n].z, codes[n].w};
                            const uint32_t sc = scale_bits<T>(exps[n]) * 0x10001u;
                            uint32_t o[8];
#pragma unroll
                            for (int k = 0; k < 4; ++k) codes_to_pairs<T>(u[k], sc, o[2 * k], o[2 * k + 1]);
                            if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                                if (exps[n] > kBigExp) {          // values beyond 57344
                                    const uint32_t more = big_scale(exps[n]) * 0x10001u;
#pragma unroll
                                    for (int k = 0; k < 8; ++k) o[k] = times_pair(o[k], more);
                                }
                            }
                            static_assert(kTile / kMine % 8 == 0, "a thread's positions are swizzled alike");
                            *reinterpret_cast<uint4 *>(dst + (n0 + n) * (kTile / kMine) * 128 + ch) = make_uint4(o[0], o[1], o[2], o[3]);
                            *reinterpret_cast<uint4 *>(dst + (n0 + n) * (kTile / kMine) * 128 + (ch ^ 16)) = make_uint4(o[4], o[5], o[6], o[7]);
                        }
                    }
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(&sh.full[s]);
                        mbar_arrive(&sh.raw_empty[rs]);
                    }
                }
                job_done(i);
            }
            if (!ok && lane == 0) report_timeout(a.kv.status);
        }
    }
    tc_fence_before();
    __syncwarp();
    cluster_wait();
    if (a.ctas > 1) cluster_sync_all();                     // nobody leaves while a neighbour may write to its shared memory
    else __syncthreads();
    if (warp == 3) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

template <typename T, bool Q8, int D>
cudaError_t launch(const CUtensorMap &q_map, const CUtensorMap &k_map, const CUtensorMap &v_map, const AttendArgs &a, int sms,
                   cudaStream_t stream)
{
    const cudaError_t e = cudaFuncSetAttribute(attend_umma_kernel<T, Q8, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    if (e != cudaSuccess) return e;
    return launch_workers(attend_umma_kernel<T, Q8, D>, Geometry<Q8, D>::kThreads, kSmemBytes, a.ctas, sms, stream, q_map, k_map, v_map, a);
}

}  // namespace

size_t attend_umma_part_floats(int sms, int d) { return (size_t)sms * 2 * part_floats(d); }

cudaError_t launch_attend_umma(const CUtensorMap &q_map, const CUtensorMap &k_map, const CUtensorMap &v_map,
                               const AttendArgs &args, int sms, cudaStream_t stream)
{
    AttendArgs a = args;
    if (a.wait_cycles <= 0) a.wait_cycles = kWaitCycles;
    // One row tile per sequence and head (the hint says), and no more of them than half the SMs: clusters share them (101 rows of 32
    // heads at 1999 positions 23.6 us, without clusters 29.0).  No more CTAs than give every stream a tile of the longest sequence that
    // the table can hold.
    const long long items = (long long)a.kv.B * a.kv.heads, tiles = (((long long)a.kv.width << a.kv.page_shift) + kTile - 1) / kTile;
    long long ctas = a.max_chunk <= kTile / a.group ? sms / items : 1;
    if (ctas > (tiles + 1) / 2) ctas = (tiles + 1) / 2;
    a.ctas = ctas >= 4 ? 4 : ctas >= 2 ? 2 : 1;       // (a power of two divides the octets of a row)
    a.tile_tokens = kTile / a.group;
    a.by_rows = FastDiv(a.ctas > 1 ? a.tile_tokens : 2 * a.tile_tokens);
    a.by_unit = FastDiv(2 * a.ctas);
    a.groups = 1;
    a.fixed = kFixed;
    a.small = plan_is_small(a, kTile / a.group * a.group, tiles + 1);
    const bool q8 = a.kv.k_exps != nullptr;
    if (a.kv.dtype == kF16) {
        if (a.kv.d == 64) return q8 ? launch<__half, true, 64>(q_map, k_map, v_map, a, sms, stream) : launch<__half, false, 64>(q_map, k_map, v_map, a, sms, stream);
        return q8 ? launch<__half, true, 128>(q_map, k_map, v_map, a, sms, stream) : launch<__half, false, 128>(q_map, k_map, v_map, a, sms, stream);
    }
    if (a.kv.d == 64) return q8 ? launch<__nv_bfloat16, true, 64>(q_map, k_map, v_map, a, sms, stream) : launch<__nv_bfloat16, false, 64>(q_map, k_map, v_map, a, sms, stream);
    return q8 ? launch<__nv_bfloat16, true, 128>(q_map, k_map, v_map, a, sms, stream) : launch<__nv_bfloat16, false, 128>(q_map, k_map, v_map, a, sms, stream);
}

}  // namespace dresd
