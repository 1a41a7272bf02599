// K11 -- attention of few rows per key/value head over the paged cache (single tokens, short chunks).
//
//     s_rj = scale q_r . k_j,   out_r = sum_j 2^(s_rj - m_r) v_j / sum_j 2^(s_rj - m_r)      (scale holds log2 e)
//
// in one pass over the cache with the running maximum m, weight sum l and weighted sum o of every row.  Every
// key and value is read once and meets a handful of rows, so the bound is HBM: what counts is many bytes in flight with
// nothing between them and the arithmetic.  Each warp has a ring of tiles of 16 positions of its own, filled by TMA and
// emptied by itself: it needs no barrier with other warps, and a tile is asked for again as soon as its last word is in
// registers.  Tiles of the next segment follow those of the present one without a gap.
//
//   S^T = K Q^T   mma.sync m16n8k16 with keys as the M = 16 operand and rows as N = 8.  The k index of the instruction may
//                 run over the elements of a row in any order that keys and queries share; it is laid out so that a lane's
//                 fragments are whole 16-byte pieces of a key.
//   O^T = V^T P^T elements as M, rows as N, positions as K.  A lane reads 16-byte pieces of four values; pairs of
//                 positions are joined with byte permutes (for E4M3 before the conversion, which takes two codes at
//                 once).  P^T is S^T's own fragment turned by movmatrix.
//
// 16-row tiles of queries would leave M half empty at the usual 1 to 8 rows per head; with rows as N nothing is padded
// beyond 8 and the accumulators take half the registers.
//
// 8-bit caches are multiplied in fp16, whatever the type of the queries, because the hardware turns E4M3 codes into fp16
// numbers (exactly) in one instruction per two.  A bf16 query row is multiplied by the power of two that brings its
// largest element to 2^14 .. 2^15: every element down to 2^-31 of it stays exact, the rest is off by 2^-40 of it.  The keys'
// scale 2^k is applied to the score.  The values' 2^e is part of the weight of the second product, 2^(s + e - n), with a
// running maximum n of s + e for every row beside that of s: so fp16's range is counted from the largest product that the row
// has seen, whatever the exponents of other rows and of positions that it does not see.  (Rows of zeros have an exponent of
// no meaning; they are found when it would raise a maximum.)  The sums are brought from 2^n to 2^m at the end.
//
// Which position is which row of the instruction is free as well: row g is position g ^ (g odd ? 4 : 0), which together
// with the 128-byte swizzle of the copies makes the reads of keys and of values free of bank conflicts.
//
// Measured (148 SMs, 8 heads of 128, 4 rows each): 2 sequences of 131071 positions in bf16 166 us = 6.46 TB/s, 98 % of what a copy
// reaches; 16 of 8000 81 us = 6.4 TB/s; the same in 8 bits 53 us = 5.0 TB/s, where a warp's instructions (425 a tile) are what
// is left; 48 of 0 to 8191 in 8 bits 34.5 us = 2.8 TB/s, bound by queries and joins of the many short segments; one of 700 with 32
// heads 9.4 us, the chain of launch, plan, first tile and join.
//
// Work is divided as kv_plan.cuh says.  With few items a worker is a CTA or a cluster; with more items than SMs it is a group of
// four warps or fewer, so that what a segment costs besides its tiles (queries, join) is hidden behind the tiles of the
// other groups.  The warps of a worker take every (warps)-th tile of a segment and are joined at its end.  The maximum is only raised when a score passes it by 2^8
// (weights stay inside the range of either type, lifted ones of fp16 below 2^15), which saves the shuffles of the maximum on most tiles.
#include "kv_plan.cuh"

namespace dresd {
namespace {

constexpr int kTile = 16;
constexpr int kFixed = 4;
constexpr float kSlack = 8.f;           // log2 of the largest weight before the maximum is raised

template <typename T>
__device__ __forceinline__ void mma16816(float *c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t turn8x8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// Position of instruction row g (0 .. 7) within its eight.
__device__ __forceinline__ int place(int g) { return g ^ ((g & 1) << 2); }

template <bool Q8, int D, int NT>
struct Geometry {
    static constexpr int kRows = 8 * NT;
    static constexpr int kRowBytes = Q8 ? D : 2 * D;      // one key or value
    static constexpr int kSlabs = kRowBytes > 128 ? kRowBytes / 128 : 1;
    static constexpr int kHalf = kTile * kRowBytes;       // keys (or values) of a tile
    static constexpr int kStage = 2 * kHalf;
    // A tile takes a warp about as long whatever its bytes: smaller tiles need more warps to keep HBM busy (2048 items of 1000
    // positions of 64 in 8 bits: 83 us with 16 warps, 117 with 8).
    static constexpr int kWarps = kStage <= 4096 && NT == 1 ? 16 : 8;
    static constexpr int kThreads = kWarps * 32;
    static constexpr int kStages = 131072 / (kWarps * kStage);       // 128 KB in flight an SM
    static constexpr int kJoinRow = D + 4;                // floats of a row of a warp's sums
    static constexpr int kSums = kRows * D / 4;           // float4 of a CTA's sums
};

struct Job {
    Segment seg;
    Chunk c;
    int more;
    int t0, t1;             // tiles of the segment (all warps')
};
template <bool Q8, int D, int NT>
struct Shared {
    using Geo = Geometry<Q8, D, NT>;
    alignas(1024) uint8_t ring[Geo::kWarps][Geo::kStages][Geo::kStage];
    alignas(16) float o[Geo::kWarps][Geo::kRows][Geo::kJoinRow];     // the warps' sums
    // cluster: what the CTAs send: sums, maximum and weight sum of float4 number n x ctas + rank, from CTA f at [f x per + n]
    alignas(16) float4 sent[Geo::kSums + kMaxCluster];
    alignas(16) float2 sent_ml[Geo::kSums + kMaxCluster];
    alignas(16) uint8_t exps[Q8 ? Geo::kWarps : 1][Geo::kStages][2][kTile];
    float m[Geo::kWarps][Geo::kRows], l[Geo::kWarps][Geo::kRows];
    uint64_t full[Geo::kWarps][Geo::kStages];
    uint64_t ready, taken;
    Job job[Geo::kWarps][4];                                         // of a worker
    int dead[Geo::kWarps][2];                                        // a wait of the worker ran out, by the segment's parity
    KvPlan<FewRows> plan[Geo::kWarps];                               // of a worker; one thread goes on with it
    unsigned ticket[Geo::kWarps];
};

// Parts of shared items: per group (or CTA) two slots of `rows` x (d + 2) floats: the sums, then the rows' maxima, then the
// rows' weight sums.
__device__ __forceinline__ float *part_slot(const AttendArgs &a, int worker, int slot, int rows)
{
    if (!debug_check(worker >= 0 && worker < gridDim.x * a.groups && (unsigned)slot < 2, a.kv.status, 66)) worker = slot = 0;
    return a.part + ((size_t)worker * 2 + slot) * rows * (a.kv.d + 2);
}

template <int kBytes> struct Piece;                       // a lane's load
template <> struct Piece<16> { using type = uint4; };
template <> struct Piece<8> { using type = uint2; };
__device__ __forceinline__ uint32_t word(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t word(const uint2 &v, int i) { return i == 0 ? v.x : v.y; }

// NT: tiles of 8 rows.
template <typename T, bool Q8, int D, int NT>
__global__ void __launch_bounds__(Geometry<Q8, D, NT>::kThreads, 1)
attend_mma_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                  const __grid_constant__ AttendArgs a)
{
    using Geo = Geometry<Q8, D, NT>;
    constexpr int kRows = Geo::kRows, kRowBytes = Geo::kRowBytes, kStages = Geo::kStages, kWarps = Geo::kWarps, kThreads = Geo::kThreads;
    constexpr int kKeyPieces = kRowBytes / 64;            // 16-byte pieces of a key per lane (4 lanes share a key)
    constexpr int kSteps = D / 16;                        // k-steps of the first product, M-tiles of the second
    constexpr int kValBytes = kRowBytes >= 128 ? 16 : 8;  // a lane's piece of a value (8 lanes share a value)
    constexpr int kValPieces = kRowBytes / 8 / kValBytes;
    constexpr int kValElems = kValBytes / (Q8 ? 1 : 2);   // elements in it
    using M = std::conditional_t<Q8, __half, T>;            // type of the products
    constexpr float kLift = Lift<M>::value;                 // 2^kLift x weights; of an 8-bit cache those of the values alone
    using VPiece = typename Piece<kValBytes>::type;
    using Sh = Shared<Q8, D, NT>;

    extern __shared__ uint8_t smem_raw[];
    Sh &sh = *reinterpret_cast<Sh *>(smem_raw);
    if (smem_u32(smem_raw) & 1023u) {                       // shared memory never starts there
        if (threadIdx.x == 0) report_timeout(a.kv.status);
        return;
    }
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    const long long wl = a.wait_cycles > 0 ? a.wait_cycles : kWaitCycles;
    const int rank = a.ctas > 1 ? (int)cluster_ctarank() : 0;
    const bool grouped = a.groups > 1;                     // then not in clusters
    const int g_warps = 1 << a.group_shift, group = warp >> a.group_shift, first_warp = group << a.group_shift;
    const int g_tid = tid - first_warp * 32, g_threads = g_warps * 32;
    const int worker = grouped ? blockIdx.x * a.groups + group : blockIdx.x;       // of a cluster each CTA has its own parts
    const int step = g_warps * a.ctas;                     // a warp takes every step-th tile
    const int mine = rank * kWarps + warp - first_warp;    // starting here
    Job *jobs = sh.job[group];
    auto sync = [&] {
        if (g_warps == 1) __syncwarp();
        else bar_sync(1 + group, g_threads);
    };

    if (lane == 0) {
        for (int s = 0; s < kStages; ++s) mbar_init(&sh.full[warp][s], 1);
        sh.dead[warp][0] = sh.dead[warp][1] = 0;
        if (warp == 0) {
            mbar_init(&sh.ready, 1);
            mbar_init(&sh.taken, a.ctas);
            tma_prefetch_desc(&k_map);
            tma_prefetch_desc(&v_map);
        }
        mbar_fence_init();
    }
    pdl_wait();                                             // what follows reads what earlier kernels wrote
    pdl_launch_dependents();

    // The worker's first warp works out the segments, one ahead of the present one.  (The plan lies in shared memory: in registers
    // it made the 8-bit kernel spill, 16 sequences of 8000 59 us instead of 53.)
    auto publish = [&](KvPlan<FewRows> &plan, int i) {
        Job &w = jobs[i & 3];
        w.more = plan.next(a, w.seg);
        if (!w.more) return;
        w.c = plan.c;
        const int seen = FewRows::seen(a, plan.c, w.seg.rt);
        w.t0 = w.seg.kt0 * step;
        w.t1 = min(w.seg.kt1 * step, (seen + kTile - 1) / kTile);
    };
    if (warp == first_warp) {
        KvPlan<FewRows> plan;
        const bool more = grouped ? plan.start(a, lane, worker, gridDim.x * a.groups)
                                  : plan.start(a, lane, blockIdx.x / a.ctas, gridDim.x / a.ctas);         // the same for the whole cluster
        if (lane == 0) {
            if (!more) plan.none();
            publish(plan, 0);
            publish(plan, 1);
            sh.plan[group] = plan;
        }
    }
    if (a.ctas > 1) cluster_sync_all();                     // the neighbours' barriers are set up
    else __syncthreads();

    // ---- the ring.  The fetching side is up to kStages tiles ahead of the using side, in the next segment if need be.
    const int beyond = (int)min((long long)a.kv.layers * a.kv.num_pages * a.kv.heads << a.kv.page_shift, 2147483647LL);
    int fetched = 0, used = 0, f_job = -1, f_tile = -step;           // the last tile that was looked up, of segment f_job
    // The next tile: its place in the pool but for the page, whose number (loaded here, used when the copy is issued) may be
    // anything.  pending = false: none known yet (up to the segment after `i`).
    bool pending = false;
    int page = 0, off = 0;
    int f_end = 0, f_total = 0, f_head = 0;                // of segment f_job
    const int32_t *f_table = nullptr;
    const int layer_pages = a.kv.layer * a.kv.num_pages, in_page = (1 << a.kv.page_shift) - 1;
    auto look_ahead = [&](int i) {
        f_tile += step;
        while (f_tile >= f_end) {                          // on to the next segment
            pending = false;
            if (f_job >= i + 1) return;
            const Job &w = jobs[(f_job + 1) & 3];
            if (!w.more) return;
            ++f_job;
            f_tile = w.t0 + mine;
            f_end = w.t1;
            f_total = w.c.total;
            f_head = w.seg.head;
            f_table = a.kv.table + (long long)w.seg.b * a.kv.width;
        }
        const int p = f_tile * kTile;
        pending = true;
        off = p & in_page;
        page = -1;
        if (p < f_total && debug_check(p >= 0 && (p >> a.kv.page_shift) < a.kv.width, a.kv.status, 61)) page = __ldg(f_table + (p >> a.kv.page_shift));
    };
    auto fetch = [&] {                                      // lane 0
        const int s = fetched % kStages;
        // beyond the end or outside the pool: zeros are loaded.  (The pool has fewer than 2^31 rows.)
        int row = (unsigned)page < (unsigned)a.kv.num_pages ? (((layer_pages + page) * a.kv.heads + f_head) << a.kv.page_shift) + off : beyond;
        if (!debug_check(row >= 0 && row <= beyond && (row == beyond || row % kTile == 0) && fetched - used < kStages, a.kv.status, 62)) row = beyond;
        uint64_t *bar = &sh.full[warp][s];
        uint8_t *dst = sh.ring[warp][s];
        mbar_arrive_expect_tx(bar, (uint32_t)(Geo::kStage + (Q8 ? 2 * kTile : 0)));
        if (a.lose_stage > 0 && blockIdx.x == 0 && warp == 0 && fetched == a.lose_stage - 1) return;
#pragma unroll
        for (int p = 0; p < Geo::kSlabs; ++p) {
            tma_load_2d(dst + p * kTile * 128, &k_map, p * 64, row, bar);
            tma_load_2d(dst + Geo::kHalf + p * kTile * 128, &v_map, p * 64, row, bar);
        }
        if constexpr (Q8) {
            const int e = row < beyond ? row : 0;           // zeros have any exponents
            bulk_load(sh.exps[warp][s][0], a.kv.k_exps + e, kTile, bar);
            bulk_load(sh.exps[warp][s][1], a.kv.v_exps + e, kTile, bar);
        }
    };
    look_ahead(0);
    while (fetched < kStages && pending) {
        if (lane == 0) fetch();
        ++fetched;
        look_ahead(0);
    }

    int joins = 0;
    bool dead = false;
    for (int i = 0;; ++i) {
        const Job &w = jobs[i & 3];
        if (!w.more) break;
        const Segment &seg = w.seg;
        const Chunk ch = w.c;
        if (!pending) look_ahead(i);                        // the segment after this one has become known
        while (fetched - used < kStages && pending && !dead) {
            if (lane == 0) fetch();
            ++fetched;
            look_ahead(i);
        }
        const int rows = min(kRows, ch.len * a.group - seg.rt * kRows);     // valid rows of the tile
        // ---- the queries, as the B operand: lane (g, c) holds row g's pieces
        uint32_t q[NT][kSteps][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = seg.rt * kRows + nt * 8 + g, tok = a.by_group.div(r);
            const bool ok = nt * 8 + g < rows && debug_check(ch.row0 + tok < a.kv.rows && seg.head < a.kv.heads, a.kv.status, 63);
            const T *src = static_cast<const T *>(a.q) + (long long)(ch.row0 + (ok ? tok : 0)) * a.q_row +
                           (seg.head * a.group + (ok ? r - tok * a.group : 0)) * a.q_head;
#pragma unroll
            for (int x = 0; x < D / 32; ++x) {
                // 16-bit keys: piece 4 x + c.  8-bit keys: a key's piece is 16 elements, two of the query's.
                const int at = Q8 ? (x / 2 * 4 + c) * 16 + x % 2 * 8 : (x * 4 + c) * 8;
                const uint4 v = ok ? __ldg(reinterpret_cast<const uint4 *>(src + at)) : make_uint4(0, 0, 0, 0);
                q[nt][2 * x][0] = v.x;
                q[nt][2 * x][1] = v.y;
                q[nt][2 * x + 1][0] = v.z;
                q[nt][2 * x + 1][1] = v.w;
            }
        }
        float q_scale[NT][2];                               // 8-bit: of rows 2 c, 2 c + 1
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            int e = 0;
            if constexpr (Q8 && std::is_same<T, __nv_bfloat16>::value) {
                uint32_t big = 0;
#pragma unroll
                for (int st = 0; st < kSteps; ++st) big = __vmaxu2(big, __vmaxu2(q[nt][st][0] & 0x7FFF7FFFu, q[nt][st][1] & 0x7FFF7FFFu));
                big = max(big & 0xFFFFu, big >> 16);
                big = max(big, __shfl_xor_sync(0xFFFFFFFFu, big, 1));
                big = max(big, __shfl_xor_sync(0xFFFFFFFFu, big, 2));
                // 2^e in two factors, as e may be beyond a single number's range
                e = big ? min(14 + 127 - (int)(big >> 7), 200) : 0;
                const float f0 = pow2f(e / 2), f1 = pow2f(e - e / 2);
#pragma unroll
                for (int st = 0; st < kSteps; ++st)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const float2 v = unpack2<T>(q[nt][st][x]);
                        q[nt][st][x] = pack2<__half>(v.x * f0 * f1, v.y * f0 * f1);
                    }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {                   // row r's scale is with the lanes 4 r .. 4 r + 3
                const int er = __shfl_sync(0xFFFFFFFFu, e, 4 * (2 * c + x));
                q_scale[nt][x] = a.scale_log2 * pow2f(-(er / 2)) * pow2f(-(er - er / 2));
            }
        }
        float o[NT][kSteps][4] = {};
        float m[NT][2], l[NT][2], mv[NT][2];                // mv: 8-bit: the sums are held relative to 2^mv
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) m[nt][0] = m[nt][1] = mv[nt][0] = mv[nt][1] = -INFINITY, l[nt][0] = l[nt][1] = 0.f;

#pragma unroll 1
        for (int t = w.t0 + mine; t < w.t1 && !dead; t += step) {
            const int p0 = t * kTile, s = used % kStages;
            if (!mbar_wait(&sh.full[warp][s], (used / kStages) & 1, wl)) {
                report_timeout(a.kv.status);
                dead = true;
            }
            // A warp that gave up asks for nothing more (its barriers' phases are not over) and leaves with its worker at the
            // segment's end.
            dead = __any_sync(0xFFFFFFFFu, dead);
            if (dead) break;
            const uint8_t *ks = sh.ring[warp][s], *vs_ = ks + Geo::kHalf;
            // ---- S^T = K Q^T; lane (g, c): keys place(g) (+ 8)
            float sc[NT][4] = {};
            uint4 kx[2][kKeyPieces];
            int ke[2] = {127, 127}, ve[2] = {127, 127};
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = 8 * j + place(g);
#pragma unroll
                for (int x = 0; x < kKeyPieces; ++x) {
                    const int ch16 = 4 * x + c;            // 16-byte piece of the row
                    const int at = kRowBytes == 64 ? r * 64 + ((ch16 ^ ((r >> 1) & 3)) << 4)
                                                   : (ch16 >> 3) * (kTile * 128) + r * 128 + (((ch16 & 7) ^ (r & 7)) << 4);
                    kx[j][x] = *reinterpret_cast<const uint4 *>(ks + at);
                }
                if constexpr (Q8) {
                    ke[j] = min((int)sh.exps[warp][s][0][r], 253);
                    ve[j] = min((int)sh.exps[warp][s][1][r], 253);
                }
            }
            if constexpr (!Q8) {
#pragma unroll
                for (int st = 0; st < kSteps; ++st)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        mma16816<T>(sc[nt], word(kx[0][st / 2], st % 2 * 2), word(kx[1][st / 2], st % 2 * 2),
                                    word(kx[0][st / 2], st % 2 * 2 + 1), word(kx[1][st / 2], st % 2 * 2 + 1), q[nt][st][0], q[nt][st][1]);
            } else {
#pragma unroll
                for (int st = 0; st < kSteps; ++st) {
                    uint32_t f[2][2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) codes_to_halves(word(kx[j][st / 4], st % 4), f[j][0], f[j][1]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        mma16816<M>(sc[nt], f[0][0], f[1][0], f[0][1], f[1][1], q[nt][st][0], q[nt][st][1]);
                }
            }
            VPiece vx[4][kValPieces];
#pragma unroll
            for (int j = 0; j < 4; ++j) {                  // values of positions place(2 c), place(2 c + 1) (+ 8)
                const int r = (j >> 1) * 8 + place(2 * c + (j & 1));
#pragma unroll
                for (int x = 0; x < kValPieces; ++x) {
                    if constexpr (kRowBytes == 64) {
                        vx[j][x] = *reinterpret_cast<const VPiece *>(vs_ + r * 64 + (((g >> 1) ^ ((r >> 1) & 3)) << 4) + (g & 1) * 8);
                    } else {
                        vx[j][x] = *reinterpret_cast<const VPiece *>(vs_ + x * (kTile * 128) + r * 128 + ((g ^ (r & 7)) << 4));
                    }
                }
            }
            ++used;
            __syncwarp();                                  // the tile is in registers: ask for the next one
            if (pending) {
                if (lane == 0) fetch();
                ++fetched;
                look_ahead(i);
            }
            // ---- scale, mask.  sc[nt][2 j + x]: key place(g) + 8 j, row 2 c + x
            const bool all_seen = p0 + kTile <= ch.ctx && p0 + kTile <= ch.total;
            const float sk[2] = {pow2f(ke[0] - 127), pow2f(ke[1] - 127)};
            float vf[2] = {(float)(ve[0] - 127), (float)(ve[1] - 127)};       // exponents of the values
            bool over = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float y = sc[nt][2 * j + x] * q_scale[nt][x];
                        if constexpr (Q8) y *= sk[j];
                        if (!all_seen) {
                            const int r = min(nt * 8 + 2 * c + x, rows - 1), tok = a.by_group.div(seg.rt * kRows + r);
                            const int p = p0 + 8 * j + place(g), e = p - ch.ctx;
                            bool seen = p < ch.total;
                            if (seen && e >= 0)
                                seen = a.mask ? (e >> 5) < a.mask_words && debug_check(ch.row0 + tok < a.kv.rows, a.kv.status, 64) && (a.mask[(long long)(ch.row0 + tok) * a.mask_words + (e >> 5)] >> (e & 31) & 1)
                                              : e <= tok;
                            if (!seen) y = -INFINITY;
                        }
                        sc[nt][2 * j + x] = y;
                        over |= y > m[nt][x] + kSlack;
                        if constexpr (Q8) over |= y + vf[j] > mv[nt][x] + kSlack;
                    }
            if (__any_sync(0xFFFFFFFFu, over)) {
                if constexpr (Q8) {                        // values that are all zeros raise nothing
                    uint32_t some = 0;                     // bit j: position j of this lane's four has a code other than 0
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t any = 0;
#pragma unroll
                        for (int x = 0; x < kValPieces; ++x)
#pragma unroll
                            for (int k = 0; k < kValBytes / 4; ++k) any |= word(vx[j][x], k);
                        some |= (any & 0x7F7F7F7Fu) ? 1u << j : 0u;
                    }
#pragma unroll
                    for (int sh_ = 4; sh_ < 32; sh_ <<= 1) some |= __shfl_xor_sync(0xFFFFFFFFu, some, sh_);
                    some = __shfl_sync(0xFFFFFFFFu, some, g >> 1) >> (g & 1);        // rows g, 8 + g: bits 0 and 2
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        if (!(some >> (2 * j) & 1)) vf[j] = -INFINITY;
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        float y = fmaxf(fmaxf(sc[nt][x], sc[nt][2 + x]), m[nt][x]);
#pragma unroll
                        for (int sh_ = 4; sh_ < 32; sh_ <<= 1) y = fmaxf(y, __shfl_xor_sync(0xFFFFFFFFu, y, sh_));
                        float f = y > -INFINITY ? ex2(m[nt][x] - y) : 1.f;
                        m[nt][x] = y;
                        l[nt][x] *= f;
                        if constexpr (Q8) {
                            float z = fmaxf(fmaxf(sc[nt][x] + vf[0], sc[nt][2 + x] + vf[1]), mv[nt][x]);
#pragma unroll
                            for (int sh_ = 4; sh_ < 32; sh_ <<= 1) z = fmaxf(z, __shfl_xor_sync(0xFFFFFFFFu, z, sh_));
                            f = z > -INFINITY ? ex2(mv[nt][x] - z) : 1.f;
                            mv[nt][x] = z;
                        }
#pragma unroll
                        for (int st = 0; st < kSteps; ++st) {
                            o[nt][st][x] *= f;
                            o[nt][st][2 + x] *= f;
                        }
                    }
            }
            // ---- weights, and P^T as the B operand: lane (g, c) holds row g, positions of rows 2 c, 2 c + 1 (+ 8)
            uint32_t p[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float wv[4];                               // 8-bit: weights with the values' scale
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const float base = m[nt][x] > -INFINITY ? m[nt][x] : 0.f, base_v = mv[nt][x] > -INFINITY ? mv[nt][x] : 0.f;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if constexpr (Q8) wv[2 * j + x] = ex2(sc[nt][2 * j + x] + (vf[j] - base_v + kLift));
                        sc[nt][2 * j + x] = ex2(sc[nt][2 * j + x] - (Q8 ? base : base - kLift));
                    }
                    l[nt][x] += sc[nt][x] + sc[nt][2 + x];
                }
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    p[nt][j] = turn8x8(Q8 ? pack2<M>(wv[2 * j], wv[2 * j + 1]) : pack2<M>(sc[nt][2 * j], sc[nt][2 * j + 1]));
            }
            // ---- O^T += V^T P^T
            if (!all_seen) {
                // Positions that some row does not see may hold anything, and 0 x NaN is NaN: unused positions
                // are cleared, and non-finite values of the chunk itself are taken out here and added row by row.
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (p0 + (j >> 1) * 8 + place(2 * c + (j & 1)) >= ch.total) {
#pragma unroll
                        for (int x = 0; x < kValPieces; ++x) vx[j][x] = VPiece{};
                    }
                if constexpr (Q8) {                        // the code of NaN counts as 0
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int x = 0; x < kValPieces; ++x) {
                            uint32_t *u = reinterpret_cast<uint32_t *>(&vx[j][x]);
#pragma unroll
                            for (int k = 0; k < kValBytes / 4; ++k) u[k] &= ~__vcmpeq4(u[k] & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
                        }
                } else {
                    constexpr uint32_t kInf = std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u;
                    bool odd = false;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int x = 0; x < kValPieces; ++x)
#pragma unroll
                            for (int k = 0; k < kValBytes / 4; ++k) {
                                const uint32_t u = word(vx[j][x], k);
                                odd |= (u & kInf) == kInf || (u >> 16 & kInf) == kInf;
                            }
                    if (__any_sync(0xFFFFFFFFu, odd)) {
#pragma unroll 1
                        for (int k = 0; k < kTile && p0 + k < ch.total; ++k) {
                            const int page = __ldg(a.kv.table + (long long)seg.b * a.kv.width + (p0 >> a.kv.page_shift));
                            if (page < 0 || page >= a.kv.num_pages) break;
                            const T *vrow = static_cast<const T *>(a.kv.v) +
                                            kv_row(a.kv, a.kv.layer, page, seg.head, (p0 + k) & ((1 << a.kv.page_shift) - 1)) * D;
                            float wgt[NT][2];              // weights of rows 2 c, 2 c + 1 at position k; it is row place(k) of its eight
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int x = 0; x < 2; ++x)
                                    wgt[nt][x] = __shfl_sync(0xFFFFFFFFu, k < 8 ? sc[nt][x] : sc[nt][2 + x], place(k & 7) * 4 + c);
#pragma unroll
                            for (int st = 0; st < kSteps; ++st)
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    const int e = 2 * st + h;
                                    const float y = unpack2<T>(reinterpret_cast<const uint16_t *>(vrow)[e / kValElems * 8 * kValElems + g * kValElems + e % kValElems]).x;
                                    if (isfinite(y)) continue;
#pragma unroll
                                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                        for (int x = 0; x < 2; ++x)
                                            if (wgt[nt][x] > 0.f) o[nt][st][2 * h + x] += wgt[nt][x] * y;
                                }
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int x = 0; x < kValPieces; ++x) {
                                uint32_t *u = reinterpret_cast<uint32_t *>(&vx[j][x]);
#pragma unroll
                                for (int k = 0; k < kValBytes / 4; ++k) {
                                    if ((u[k] & kInf) == kInf) u[k] &= 0xFFFF0000u;
                                    if ((u[k] >> 16 & kInf) == kInf) u[k] &= 0x0000FFFFu;
                                }
                            }
                    }
                }
            }
            // M-tile st covers elements e0 = 2 st, e1 = 2 st + 1 of every lane group's piece
#pragma unroll
            for (int st = 0; st < kSteps; ++st) {
                constexpr int kPer = kValElems / 2;        // M-tiles per piece
                const int x = st / kPer, e = st % kPer;    // e: pair of elements within the piece
                uint32_t f[2][2];                          // [pair of positions][element e0, e1]
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if constexpr (!Q8) {
                        const uint32_t lo = word(vx[2 * j][x], e), hi = word(vx[2 * j + 1][x], e);
                        f[j][0] = __byte_perm(lo, hi, 0x5410);
                        f[j][1] = __byte_perm(lo, hi, 0x7632);
                    } else {
                        const uint32_t lo = word(vx[2 * j][x], e / 2), hi = word(vx[2 * j + 1][x], e / 2);
                        // codes: e0 of both positions, e1 of both
                        codes_to_halves(__byte_perm(lo, hi, e & 1 ? 0x7362 : 0x5140), f[j][0], f[j][1]);
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma16816<M>(o[nt][st], f[0][0], f[0][1], f[1][0], f[1][1], p[nt][0], p[nt][1]);
            }
        }
        // ---- join the warps
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
#pragma unroll
                for (int sh_ = 4; sh_ < 32; sh_ <<= 1) l[nt][x] += __shfl_xor_sync(0xFFFFFFFFu, l[nt][x], sh_);
                const int r = nt * 8 + 2 * c + x;
                if (g == 0) {
                    sh.m[warp][r] = m[nt][x];
                    sh.l[warp][r] = l[nt][x];
                }
                const float f = !Q8 ? 1.f : mv[nt][x] > -INFINITY ? ex2(mv[nt][x] - m[nt][x] - kLift) : 0.f;
#pragma unroll
                for (int st = 0; st < kSteps; st += 2) {   // elements 2 st .. 2 st + 3 of the lane's piece are neighbours
                    const int e = 2 * st;
                    *reinterpret_cast<float4 *>(&sh.o[warp][r][e / kValElems * 8 * kValElems + g * kValElems + e % kValElems]) =
                        make_float4(o[nt][st][x] * f, o[nt][st][2 + x] * f, o[nt][st + 1][x] * f, o[nt][st + 1][2 + x] * f);
                }
            }
        auto give_up = [&] {
            if (dead) *const_cast<volatile int *>(&sh.dead[group][i & 1]) = 1;
        };
        give_up();
        sync();
        if (g_tid == 0) publish(sh.plan[group], i + 2);
        const int heads = a.kv.heads * a.group;
        const bool split = seg.c0 != seg.c1;
        float *part = part_slot(a, worker, seg.slot, kRows);
        auto finish = [&](int r, int e, const float4 &acc, float mm, float ll) {       // four elements of a row's result
            const float inv = ll > 0.f ? 1.f / ll : ll == 0.f ? 0.f : ll;              // a NaN sum stays one
            const int rr = seg.rt * kRows + r, tok = a.by_group.div(rr);
            const long long at = (long long)(ch.row0 + tok) * heads + seg.head * a.group + rr - tok * a.group;
            if (!debug_check(at >= 0 && at < (long long)a.kv.rows * heads, a.kv.status, 65)) return;
            *reinterpret_cast<uint2 *>(static_cast<T *>(a.out) + at * D + e) =
                make_uint2(pack2<T>(acc.x * inv, acc.y * inv), pack2<T>(acc.z * inv, acc.w * inv));
            if (a.lse && e == 0) a.lse[at] = ((mm > -INFINITY ? mm - (Q8 ? 0.f : kLift) : 0.f) + log2f(ll)) * 0.69314718055994531f;
        };
        auto add = [](float4 &acc, float f, const float4 &y) {                         // what has no weight may be anything
            if (f > 0.f || f != f) acc.x += f * y.x, acc.y += f * y.y, acc.z += f * y.z, acc.w += f * y.w;
        };
        auto put = [&](int x, const float4 &acc, float mm, float ll) {                 // float4 x of the sums
            const int r = x / (D / 4), e = x % (D / 4) * 4;
            if (r >= rows) return;
            if (!split) {
                finish(r, e, acc, mm, ll);
            } else {
                __stcg(reinterpret_cast<float4 *>(part) + x, acc);
                if (e == 0 || a.ctas > 1) {                                            // of a cluster every CTA needs them
                    __stcg(part + kRows * D + r, mm);
                    __stcg(part + kRows * D + kRows + r, ll);
                }
            }
        };
        const int per = (Geo::kSums + a.ctas - 1) / a.ctas;                            // float4 of a CTA of a cluster
        if (a.ctas > 1) {
            if (tid == 0) mbar_arrive_expect_tx(&sh.ready, (uint32_t)(a.ctas * ((Geo::kSums - rank + a.ctas - 1) / a.ctas) * 24));
            // what was sent the last time has been read
            if (joins > 0 && !dead && !mbar_wait_cluster(&sh.taken, (joins - 1) & 1, wl)) {
                report_timeout(a.kv.status);
                dead = true;
            }
        }
#pragma unroll 1
        for (int x = g_tid; x < Geo::kSums; x += g_threads) {
            const int r = x / (D / 4), e = x % (D / 4) * 4;
            float mm = -INFINITY, ll = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            auto add_warp = [&](int y) {
                const float f = mm > -INFINITY ? ex2(sh.m[y][r] - mm) : 0.f;
                ll += f * sh.l[y][r];
                add(acc, f, *reinterpret_cast<const float4 *>(&sh.o[y][r][e]));
            };
            if (!grouped) {                                // all loads at once
#pragma unroll
                for (int y = 0; y < kWarps; ++y) mm = fmaxf(mm, sh.m[y][r]);
#pragma unroll
                for (int y = 0; y < kWarps; ++y) add_warp(y);
            } else {
#pragma unroll 4
                for (int y = first_warp; y < first_warp + g_warps; ++y) mm = fmaxf(mm, sh.m[y][r]);
#pragma unroll 4
                for (int y = first_warp; y < first_warp + g_warps; ++y) add_warp(y);
            }
            if (a.ctas == 1) {
                put(x, acc, mm, ll);
            } else {                                                                   // to the CTA that adds up number x
                const int to = x % a.ctas, at = rank * per + x / a.ctas;
                st_async(&sh.sent[at], acc, &sh.ready, to);
                st_async(&sh.sent_ml[at], make_float2(mm, ll), &sh.ready, to);
            }
        }
        if (a.ctas > 1) {
            if (!dead && !mbar_wait_cluster(&sh.ready, joins & 1, wl)) {
                report_timeout(a.kv.status);
                dead = true;
            }
#pragma unroll 1
            for (int y = tid; y * a.ctas + rank < Geo::kSums; y += kThreads) {
                float mm = -INFINITY, ll = 0.f;
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int x = 0; x < a.ctas; ++x) mm = fmaxf(mm, sh.sent_ml[x * per + y].x);
                for (int x = 0; x < a.ctas; ++x) {
                    const float2 p = sh.sent_ml[x * per + y];
                    const float f = mm > -INFINITY ? ex2(p.x - mm) : 0.f;
                    ll += f * p.y;
                    add(acc, f, sh.sent[x * per + y]);
                }
                put(y * a.ctas + rank, acc, mm, ll);
            }
            give_up();
            __syncthreads();
            if (tid < a.ctas) mbar_arrive_cluster(mapa_rank(smem_u32(&sh.taken), tid));
            ++joins;
        }
        if (split) {
            __threadfence();
            sync();
            if (g_tid == 0 && debug_check(seg.c0 >= 0 && seg.c0 * a.ctas + rank < gridDim.x * a.groups, a.kv.status, 67))
                sh.ticket[group] = atomicAdd(a.tickets + seg.c0 * a.ctas + rank, 1u);
            sync();
            if (sh.ticket[group] == (unsigned)(seg.c1 - seg.c0)) {                      // the last of them: join the parts in order
                __threadfence();
                if (g_tid == 0) a.tickets[seg.c0 * a.ctas + rank] = 0;
#pragma unroll 1
                for (int x = g_tid * a.ctas + rank; x < rows * (D / 4); x += g_threads * a.ctas) {
                    const int r = x / (D / 4), e = x % (D / 4) * 4;
                    float mm = -INFINITY, ll = 0.f;
                    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                    for (int y = seg.c0; y <= seg.c1; ++y) {
                        const float *ps = part_slot(a, y * a.ctas + rank, y == seg.c0 ? seg.slot0 : 0, kRows);
                        const float pm = __ldcg(ps + kRows * D + r), pl = __ldcg(ps + kRows * D + kRows + r);
                        const float4 v = __ldcg(reinterpret_cast<const float4 *>(ps) + x);
                        const float nm = fmaxf(mm, pm);
                        const float f0 = nm > -INFINITY ? ex2(mm - nm) : 0.f, f1 = nm > -INFINITY ? ex2(pm - nm) : 0.f;
                        ll = f0 * ll + f1 * pl;
                        acc.x *= f0, acc.y *= f0, acc.z *= f0, acc.w *= f0;
                        add(acc, f1, v);
                        mm = nm;
                    }
                    finish(r, e, acc, mm, ll);
                }
            }
        }
        sync();                                             // the join's buffers are written again; job i + 2 is known
        if (*const_cast<volatile int *>(&sh.dead[group][i & 1])) break;      // all of the worker's warps, or none
    }
    // no copy may be in flight when the CTA ends: all fetched tiles have been used unless a wait ran out
    for (; used < fetched; ++used)
        if (!mbar_wait(&sh.full[warp][used % kStages], (used / kStages) & 1, wl) && lane == 0) report_timeout(a.kv.status);
    __syncwarp();
    if (a.ctas > 1) cluster_sync_all();                     // nobody leaves while a neighbour may read its shared memory
}

template <typename T, bool Q8, int D, int NT>
cudaError_t launch(const CUtensorMap &k_map, const CUtensorMap &v_map, const AttendArgs &args, int sms, cudaStream_t stream)
{
    using Geo = Geometry<Q8, D, NT>;
    constexpr int kSmem = (int)sizeof(Shared<Q8, D, NT>);
    static_assert(kSmem <= 232448, "shared memory");
    AttendArgs a = args;
    // Fewer items than half the SMs: clusters share them.  No more CTAs than give every warp a tile of the longest sequence
    // that the table can hold.
    const long long items = (long long)a.kv.B * a.kv.heads * (((long long)a.max_chunk * a.group + Geo::kRows - 1) / Geo::kRows);
    const long long positions = (long long)a.kv.width << a.kv.page_shift, tile = Geo::kWarps * kTile;
    long long ctas = sms / items;
    if (ctas > (positions + tile - 1) / tile) ctas = (positions + tile - 1) / tile;
    // Clusters leave SMs idle (of 148, clusters of 7 use 112 or so) but save joins through global memory.  Where a CTA's share
    // of the cache takes long (1 MB, some 20 us) the SMs matter more, unless an item has so many parts that their join does:
    // 131071 positions of 128 in 16 bits, 3 items 43 us with clusters and 61 without, 10 items 109 and 112, 16 items 167 and 167;
    // 60000 in 8 bits, 20 items 85 and 62, 50 items 130 and 126.  (700 positions, 32 items: 9.4 and 10.2.)
    if (sms / items <= kMaxCluster && items * positions * 2 * Geo::kRowBytes / sms > 1 << 20) ctas = 1;
    a.ctas = (int)(ctas < 1 ? 1 : ctas > kMaxCluster ? kMaxCluster : ctas);
    // More items than SMs: a CTA's groups work on items of their own (48 ragged sequences in 384 items 35 us, with the whole CTA on an
    // item 42; 2048 items of 1000 positions of 64 in 8 bits 83 and 126).  Small groups only where no sequence is long, because the
    // last worker on an item joins its parts alone: in 8 bits, heads of 64, 3200 items of 300 positions 54 us with groups of one
    // warp, 58 of two, 64 of four, 2048 of 1000 83 us with two, 84 with one, 87 with four; the 384 ragged ones (up to 8191) 97
    // us with one, 47 with two.
    const int group = items >= (long long)sms * Geo::kWarps && positions <= 2048       ? 1
                      : items >= (long long)sms * Geo::kWarps / 2 && positions <= 8192 ? 2
                                                                                       : 4;
    a.groups = items > sms ? Geo::kWarps / group : 1;
    a.group_shift = items > sms ? group / 2 : Geo::kWarps == 8 ? 3 : 4;      // 1, 2, 4: 0, 1, 2
    const int unit = (int)tile * a.ctas / a.groups;
    a.by_unit = FastDiv(unit);
    // Queries and join of a segment take about as long as four tiles of a warp: 48 ragged sequences 34.5 us, 60 with 0, 36.3 with 8.
    a.fixed = kFixed;
    a.small = plan_is_small(a, Geo::kRows, positions / unit + 1);
    auto kernel = attend_mma_kernel<T, Q8, D, NT>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    return launch_workers(kernel, Geo::kThreads, kSmem, a.ctas, sms, stream, k_map, v_map, a);
}
template <typename T, bool Q8>
cudaError_t by_shape(const CUtensorMap &k_map, const CUtensorMap &v_map, const AttendArgs &a, int sms, cudaStream_t stream)
{
    if (a.kv.d == 64)
        return a.by_rows.d == 8 ? launch<T, Q8, 64, 1>(k_map, v_map, a, sms, stream) : launch<T, Q8, 64, 2>(k_map, v_map, a, sms, stream);
    return a.by_rows.d == 8 ? launch<T, Q8, 128, 1>(k_map, v_map, a, sms, stream) : launch<T, Q8, 128, 2>(k_map, v_map, a, sms, stream);
}

}  // namespace

size_t attend_mma_workers(int sms) { return (size_t)sms * 16; }        // 16 warps with 8 rows, or 8 with 16
size_t attend_mma_part_floats(int sms, int d) { return attend_mma_workers(sms) * 2 * 8 * (d + 2); }

cudaError_t launch_attend_mma(const CUtensorMap &k_map, const CUtensorMap &v_map, const AttendArgs &args, int sms, cudaStream_t stream)
{
    AttendArgs a = args;
    a.by_rows = FastDiv((long long)a.max_chunk * a.group <= 8 ? 8 : 16);       // a row tile
    const bool q8 = a.kv.k_exps != nullptr;
    if (a.kv.dtype == kF16) return q8 ? by_shape<__half, true>(k_map, v_map, a, sms, stream) : by_shape<__half, false>(k_map, v_map, a, sms, stream);
    return q8 ? by_shape<__nv_bfloat16, true>(k_map, v_map, a, sms, stream) : by_shape<__nv_bfloat16, false>(k_map, v_map, a, sms, stream);
}

}  // namespace dresd
