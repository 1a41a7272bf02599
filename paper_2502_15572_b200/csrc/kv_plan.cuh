// Shared by the kernels of the paged key/value cache: element conversions, addresses, and the
// division of the attention's work over the CTAs.
#pragma once

#include "common.cuh"
#include "internal.h"

namespace dresd {

// ---- 8-bit rows: E4M3 codes with one power-of-two scale per (token, head) --------------------
template <typename T> struct KvType;
template <> struct KvType<__half> {
    static constexpr int kMinExp = -24;                  // 2^-24 is the finest step of fp16: a smaller scale gains nothing
    static constexpr uint32_t kBoundBits = 0x7B80u;      // 61440 = 240 x 2^8: a magnitude that is finite after rounding
};
template <> struct KvType<__nv_bfloat16> {
    static constexpr int kMinExp = -126;
    static constexpr uint32_t kBoundBits = 0x7F70u;      // 1.875 x 2^127
};

// fp16 ends at 2^-24, and a long tail of weights below that is still a part of the result: weights are held as 2^7 times what
// they are, up to 2^8 of slack over a late maximum so up to 2^15, and down to 2^-31 of the largest.  (bf16 has fp32's range.)
template <typename T> struct Lift { static constexpr float value = 0.f; };
template <> struct Lift<__half> { static constexpr float value = 7.f; };

// Least e with amax <= 448 2^e (448 = 1.75 x 2^8), from the bits of amax; 0 for amax = 0.
__device__ __forceinline__ int kv_exponent(float amax, int min_exp)
{
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return u == 0 ? 0 : max(e, min_exp);
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w)
{
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w)
{
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi)
{
    __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&h);
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi)
{
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&h);
}

// The four codes of a word as two pairs of fp16.
__device__ __forceinline__ void codes_to_halves(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    const __half2_raw x = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)w, __NV_E4M3);
    const __half2_raw y = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> 16), __NV_E4M3);
    lo = *reinterpret_cast<const uint32_t *>(&x);
    hi = *reinterpret_cast<const uint32_t *>(&y);
}
__device__ __forceinline__ uint32_t times_halves(uint32_t x, uint32_t y)
{
    const __half2 r = __hmul2(*reinterpret_cast<const __half2 *>(&x), *reinterpret_cast<const __half2 *>(&y));
    return *reinterpret_cast<const uint32_t *>(&r);
}
// The same of bf16.
__device__ __forceinline__ uint32_t times_pair(uint32_t x, uint32_t y)
{
    const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&y));
    return *reinterpret_cast<const uint32_t *>(&r);
}
// The four codes of a word as two pairs of T, times the pair `scale` = scale_bits() twice: the values, exactly.  fp16: the hardware
// conversion.  bf16: the code's bits moved to bf16's exponent and mantissa are its value x 2^-120 (the biases
// differ by 120, E4M3's subnormals become bf16's), so `scale` carries 2^120.
template <typename T>
__device__ __forceinline__ void codes_to_pairs(uint32_t w, uint32_t scale, uint32_t &lo, uint32_t &hi)
{
    if constexpr (std::is_same<T, __half>::value) {
        codes_to_halves(w, lo, hi);
        lo = times_halves(lo, scale);
        hi = times_halves(hi, scale);
    } else {
        auto moved = [](uint32_t two) { return (two & 0x80008000u) | ((two >> 4) & 0x07F007F0u); };      // codes in bytes 1 and 3
        lo = times_pair(moved(__byte_perm(w, 0, 0x1404)), scale);
        hi = times_pair(moved(__byte_perm(w, 0, 0x3424)), scale);
    }
}
// What codes_to_pairs() multiplies by for exponent byte `eb`, as the bits of one T; finite for any byte.  bf16: 2^(e + 120) is
// representable up to e = 7 (kBigExp); larger ones (values beyond 57344) are finished by a second product with big_scale().
constexpr int kBigExp = 134;
template <typename T> __device__ __forceinline__ uint32_t scale_bits(int eb);
template <> __device__ __forceinline__ uint32_t scale_bits<__half>(int eb)
{
    const int e = eb - 127;                               // -24 .. 8
    return e >= -14 ? (uint32_t)(min(e, 15) + 15) << 10 : 1u << max(e + 24, 0);
}
template <> __device__ __forceinline__ uint32_t scale_bits<__nv_bfloat16>(int eb)
{
    return (uint32_t)(min(eb, kBigExp) + 120) << 7;
}
__device__ __forceinline__ uint32_t big_scale(int eb) { return (uint32_t)(127 + max(eb - kBigExp, 0)) << 7; }

// ---- a batch of chunks -------------------------------------------------------------------------
struct Chunk {
    int row0, len;      // rows of the dense tensors
    int ctx, total;     // positions before the chunk; positions in all; both no more than the table reaches
    // Positions that token `tok` sees in causal order.  (ctx + tok may be beyond 31 bits, what the table reaches is not.)
    __device__ __forceinline__ int upto(int tok) const { return ctx + min(tok + 1, total - ctx); }
};
__device__ __forceinline__ Chunk kv_chunk(const KvArgs &a, int b)
{
    if (!debug_check(b >= 0 && b < a.B, a.status, 60)) b = 0;
    Chunk c;
    c.row0 = min(max(a.start[b], 0), a.rows);
    c.len = min(max(a.start[b + 1], c.row0), a.rows) - c.row0;
    const int reach = (int)((long long)a.width << a.page_shift);      // the host has checked that it fits
    c.ctx = min(max(a.ctx[b], 0), reach);
    c.total = c.ctx + min(c.len, reach - c.ctx);
    return c;
}
// Row of (layer, page, head, offset) in the cache arrays.
__device__ __forceinline__ long long kv_row(const KvArgs &a, int layer, int page, int head, int off)
{
    return (((((long long)layer * a.num_pages + page) * a.heads + head) << a.page_shift) + off);
}
// Rows of the cache arrays.
__device__ __forceinline__ long long kv_rows(const KvArgs &a) { return (long long)a.layers * a.num_pages * a.heads << a.page_shift; }

// ---- shared memory of the CTA and its cluster ------------------------------------------------------
constexpr int kMaxCluster = 8;

__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
// Plain bulk copy; 16-byte aligned, a multiple of 16 bytes.
__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, uint64_t *bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
                 "l"(__cvta_generic_to_global(src)), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}
// Sends to CTA `rank` of the cluster; its barrier (at the same place as `bar` here) counts the bytes when they have arrived.
__device__ __forceinline__ void st_async(float4 *p, const float4 &x, uint64_t *bar, uint32_t rank)
{
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(mapa_rank(smem_u32(p), rank)),
                 "f"(x.x), "f"(x.y), "f"(x.z), "f"(x.w), "r"(mapa_rank(smem_u32(bar), rank))
                 : "memory");
}
__device__ __forceinline__ void st_async(float2 *p, const float2 &x, uint64_t *bar, uint32_t rank)
{
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(mapa_rank(smem_u32(p), rank)),
                 "f"(x.x), "f"(x.y), "r"(mapa_rank(smem_u32(bar), rank))
                 : "memory");
}
// Bounded wait on a barrier that other CTAs of the cluster arrive on.
__device__ __forceinline__ bool mbar_wait_cluster(uint64_t *bar, uint32_t parity, long long limit)
{
    const long long t0 = clock64();
    while (true) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(smem_u32(bar)), "r"(parity)
            : "memory");
        if (ok) return true;
        if (clock64() - t0 > limit) return false;
    }
}
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ---- division of the attention's work -----------------------------------------------------------
// An ITEM is a tile of rows of one sequence and key/value head (row r of a chunk is head r % group of token r / group);
// its cost is the number of UNITS of positions that its rows see (at least one, so that every row is written).  How many
// rows and positions that is, a kernel's Shape says.  A WORKER is a CTA, or a cluster of CTAs that split every unit among
// them and join their results through shared memory.  Worker i of n gets
//
//   few items: a piece of ONE item.  With n / items workers for each, items are cut into pieces of at most L units, if L is
//       within an eighth and five units of an even share W / n: nobody starts a second item, whose queries and join cost
//       several units, and up to an eighth of the workers may idle for it (HBM is as busy without them, and an 8-bit cache,
//       which is bound by instructions, still loses more by second items).  One token at 700 positions 9.4 us, 10.4 on the
//       line; 16 at 8000, 8 heads of 128, 81 and 88, 8 bits 53 and 55 (heads of 64 43 and 45); two at 131071 166 and 165; 101 rows
//       at 1999 23.6 and 33.7.
//   otherwise: an even share of a line of all items in the order (sequence, row tile, head), so that the workers finish
//       together however ragged the batch is; a worker has the tail of one item, some whole items and the head of another.
//       An item is as long as its units and `fixed` places before them, which stand for that fixed cost.
//
// Parts of an item are joined by the worker that finishes it last, in the order of the workers, so results do not depend
// on timing.
struct Segment {
    int b, rt, head;        // the item
    int kt0, kt1;           // its units that this worker takes
    int c0, c1;             // workers that share it
    int slot;               // slot of this worker's part (0: it is the worker's first segment, 1: a later one)
    int slot0;              // slot of c0's part; those of c0 + 1 .. c1 are 0
};

// Shape of the kernel for few rows: tiles of by_rows.d rows, units of by_unit.d positions.
struct FewRows {
    static __device__ __forceinline__ int row_tiles(const AttendArgs &a, const Chunk &k) { return a.by_rows.ceil(k.len * a.group); }
    static __device__ __forceinline__ int seen(const AttendArgs &a, const Chunk &k, int r)         // positions
    {
        return a.mask ? k.total : k.upto(min(k.len - 1, a.by_group.div((r + 1) * (int)a.by_rows.d - 1)));
    }
    static __device__ __forceinline__ int units(const AttendArgs &a, const Chunk &k, int r) { return max(1, a.by_unit.ceil(seen(a, k, r))); }
};

template <typename Shape>
struct KvPlan {
    long long hi, u;            // end of this worker's part of the line; its next place
    long long even, more;       // the first `more` workers have even + 1 places, the others even
    int n;                      // workers (0: a piece each)
    int b, rt, head, kt;        // item of place u, and the place in it
    int pieces, piece;          // of the item, and this worker's
    unsigned L;                 // units of a piece
    int c0;
    bool first;
    Chunk c;

    // Units of a sequence for one head in pieces of at most L, its largest item, its row tiles.
    template <typename Int>
    static __device__ __forceinline__ Int pieces_of(const AttendArgs &a, const Chunk &k, unsigned L, unsigned *most, unsigned *items)
    {
        const int nr = Shape::row_tiles(a, k);
        Int p = 0;
        unsigned m = 0;
#pragma unroll 1
        for (int r = 0; r < nr; ++r) {
            const unsigned u = Shape::units(a, k, r);
            p += L == 1 ? u : (u + L - 1) / L;
            m = max(m, u);
        }
        *most = m;
        *items = nr;
        return p;
    }
    __device__ __forceinline__ long long begin(int i) const { return i * even + min((long long)i, more); }
    static __device__ __forceinline__ long long quotient(long long x, long long y)      // nearly always in 32 bits
    {
        return ((unsigned long long)(x | y) >> 32) == 0 ? (long long)((uint32_t)x / (uint32_t)y) : x / y;
    }
    __device__ __forceinline__ int owner(long long t) const
    {
        const long long big = more * (even + 1);
        return (int)(t < big ? quotient(t, even + 1) : more + quotient(t - big, even));
    }
    static __device__ __forceinline__ unsigned add_lanes(unsigned x) { return __reduce_add_sync(0xFFFFFFFFu, x); }
    static __device__ __forceinline__ long long add_lanes(long long x)
    {
#pragma unroll 1
        for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
        return x;
    }

    // Called by all 32 lanes of a warp of worker `me` of `count`; false = nothing to do.  A small call's time is latency, this
    // included: one pass over the lengths, and 32 bits where the host knows that they are enough.
    __device__ __forceinline__ bool start(const AttendArgs &a, int lane, int me, int count)
    {
        return a.small ? start_as<unsigned>(a, lane, me, count) : start_as<long long>(a, lane, me, count);
    }
    template <typename Int>
    __device__ bool start_as(const AttendArgs &a, int lane, int me, int count)
    {
        // a lane adds up B / 32 sequences in a row
        const int per = (a.kv.B + 31) >> 5, H = a.kv.heads, b0 = lane * per, b1 = min(b0 + per, a.kv.B);
        unsigned most = 0;
        Int own = 0, nr = 0;
#pragma unroll 1
        for (int bb = b0; bb < b1; ++bb) {
            unsigned m, i;
            own += pieces_of<Int>(a, kv_chunk(a.kv, bb), 1, &m, &i);
            most = max(most, m);
            nr += i;
        }
        most = __reduce_max_sync(0xFFFFFFFFu, most);
        const Int items = add_lanes(nr) * H, W = add_lanes(own) * H;
        first = true;
        if (W == 0) return false;
        Int find = me;
        L = 0;
        if (items <= (Int)count) {
            const unsigned each = (unsigned)count / (unsigned)items;
            L = each == 1 ? most : (most + each - 1) / each;
        }
        if (L > 0 && (Int)L * count <= W + W / 8 + 5 * count) {
            n = 0;
            if (L > 1) {
                own = 0;
#pragma unroll 1
                for (int bb = b0; bb < b1; ++bb) {
                    unsigned m, i;
                    own += pieces_of<Int>(a, kv_chunk(a.kv, bb), L, &m, &i);
                }
            }
        } else {
            L = 1;
            own += nr * a.fixed;
            const Int line = W + items * a.fixed;
            n = (int)min((Int)count, line);
            if (me >= n) return false;
            even = line / n;
            more = line - (Int)even * n;
            u = begin(me);
            hi = begin(me + 1);
            find = (Int)u;
        }
        own *= H;
        Int incl = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const Int x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += x;
        }
        const unsigned hit = __ballot_sync(0xFFFFFFFFu, incl > find);
        if (!hit) return false;
        const int l = __ffs(hit) - 1;
        Int rest = find - __shfl_sync(0xFFFFFFFFu, incl - own, l);
        b = l * per;
        c = kv_chunk(a.kv, b);
        rt = 0;
#pragma unroll 1
        while (true) {                                      // ends: the lane has more pieces than `rest`
            if (rt == Shape::row_tiles(a, c)) {
                c = kv_chunk(a.kv, ++b);
                rt = 0;
                continue;
            }
            const unsigned units = Shape::units(a, c, rt);
            pieces = n ? (int)units + a.fixed : (int)(L == 1 ? units : (units + L - 1) / L);
            if (rest < (Int)pieces * H) break;
            rest -= (Int)pieces * H;
            ++rt;
        }
        head = pieces == 1 ? (int)rest : (int)(rest / (Int)pieces);
        kt = piece = (int)(rest - (Int)head * pieces);
        c0 = me - piece;
        return true;
    }

    // A worker with nothing to do.
    __device__ __forceinline__ void none()
    {
        n = 0;
        first = false;
    }
    // The next segment; false when the worker has done its share (also when asked again).  Uniform over the worker.
    __device__ bool next(const AttendArgs &a, Segment &s)
    {
        if (n == 0) {
            if (!first) return false;
            first = false;
            s.b = b;
            s.rt = rt;
            s.head = head;
            s.kt0 = piece * (int)L;
            s.kt1 = min(Shape::units(a, c, rt), s.kt0 + (int)L);
            s.c0 = c0;
            s.c1 = c0 + pieces - 1;
            s.slot = s.slot0 = 0;
            return true;
        }
#pragma unroll 1
        while (u < hi) {
            const int size = Shape::units(a, c, rt) + a.fixed;
            if (kt == size) {                                // on to the next item (there is one: u < hi)
                kt = 0;
                if (++head < a.kv.heads) continue;
                head = 0;
                ++rt;
#pragma unroll 1
                while (rt >= Shape::row_tiles(a, c)) {
                    c = kv_chunk(a.kv, ++b);
                    rt = 0;
                }
                continue;
            }
            const long long item = u - kt;
            const int end = (int)min((long long)size, kt + (hi - u));
            s.kt0 = max(kt - a.fixed, 0);
            s.kt1 = end - a.fixed;
            u += end - kt;
            kt = end;
            if (s.kt1 <= s.kt0) continue;                    // the fixed part alone: its units are the next worker's
            s.b = b;
            s.rt = rt;
            s.head = head;
            s.c0 = owner(item + a.fixed);
            s.c1 = owner(item + size - 1);
            s.slot = first ? 0 : 1;
            s.slot0 = begin(s.c0) >= item ? 0 : 1;
            first = false;
            return true;
        }
        return false;
    }
};

// Do the plan's numbers fit 32 bits, for tiles of `rows` rows and items of at most `units` units?  start[] may contradict itself, up to
// every sequence with all rows.
inline bool plan_is_small(const AttendArgs &a, int rows, long long units)
{
    const double tiles = (double)a.kv.rows * a.group / rows + 1;
    return (double)a.kv.heads * a.kv.B * tiles * (double)(units + a.fixed) < (double)(1 << 30);
}

// A persistent kernel of one CTA per SM, as clusters of `ctas`, no more of them than the device holds at once (its SMs
// come in groups, which a cluster does not cross).
template <typename... KArgs, typename... Args>
cudaError_t launch_workers(void (*kernel)(KArgs...), int threads, int smem, int ctas, int sms, cudaStream_t stream, const Args &...args)
{
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.gridDim = dim3(sms / ctas * ctas);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = ctas > 1 ? 2 : 1;
    if (ctas > 1) {
        // by device and kernel type; every kernel of a type fills an SM
        constexpr int kDevices = 16;                        // of more than these it is asked every time
        static int held[kDevices][kMaxCluster + 1] = {};
        int device = 0;
        cudaError_t e = cudaGetDevice(&device);
        int n = e == cudaSuccess && device < kDevices ? held[device][ctas] : 0;
        if (n == 0) {
            if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
            if (e != cudaSuccess) return e;
            if (n < 1) n = 1;
            if (device < kDevices) held[device][ctas] = n;
        }
        if ((int)cfg.gridDim.x > n * ctas) cfg.gridDim.x = n * ctas;
    }
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace dresd
