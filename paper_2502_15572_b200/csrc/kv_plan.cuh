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

// Two E4M3 codes in bytes 1 and 3 of `w` (the others 0) as a pair of T, times the pair `scale`.  fp16: the hardware
// conversion.  bf16: the code's bits moved to bf16's exponent and mantissa are its value x 2^-120 (the biases
// differ by 120, E4M3's subnormals fall among the normal numbers' steps), so `scale` carries 2^120.
template <typename T> __device__ __forceinline__ uint32_t codes_to_pair(uint32_t w, uint32_t scale);
template <> __device__ __forceinline__ uint32_t codes_to_pair<__half>(uint32_t w, uint32_t scale)
{
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)__byte_perm(w, 0, 0x0031), __NV_E4M3);
    const __half2 r = __hmul2(*reinterpret_cast<const __half2 *>(&h), *reinterpret_cast<const __half2 *>(&scale));
    return *reinterpret_cast<const uint32_t *>(&r);
}
template <> __device__ __forceinline__ uint32_t codes_to_pair<__nv_bfloat16>(uint32_t w, uint32_t scale)
{
    const uint32_t b = (w & 0x80008000u) | ((w >> 4) & 0x07F007F0u);
    const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&b), *reinterpret_cast<const __nv_bfloat162 *>(&scale));
    return *reinterpret_cast<const uint32_t *>(&r);
}
// What codes_to_pair() multiplies by for exponent byte `eb`, as the bits of one T.  bf16: 2^(e + 120) is representable up
// to e = 7; larger ones (values beyond 57344) are finished by a second product with big_scale().
template <typename T> __device__ __forceinline__ uint32_t scale_bits(int eb);
template <> __device__ __forceinline__ uint32_t scale_bits<__half>(int eb)
{
    const int e = eb - 127;                               // -24 .. 8
    return e >= -14 ? (uint32_t)(min(e, 15) + 15) << 10 : 1u << max(e + 24, 0);
}
template <> __device__ __forceinline__ uint32_t scale_bits<__nv_bfloat16>(int eb)
{
    return (uint32_t)(min(eb, 134) + 120) << 7;
}
__device__ __forceinline__ uint32_t big_scale(int eb) { return (uint32_t)(127 + max(eb - 134, 0)) << 7; }


// ---- a batch of chunks -------------------------------------------------------------------------
struct Chunk {
    int row0, len;      // rows of the dense tensors
    int ctx, total;     // positions before the chunk; positions in all that the table reaches
};
__device__ __forceinline__ Chunk kv_chunk(const KvArgs &a, int b)
{
    Chunk c;
    c.row0 = min(max(a.start[b], 0), a.rows);
    c.len = min(max(a.start[b + 1], c.row0), a.rows) - c.row0;
    c.ctx = max(a.ctx[b], 0);
    c.total = (int)min((long long)c.ctx + c.len, (long long)a.width << a.page_shift);
    return c;
}
// Row of (layer, page, head, offset) in the cache arrays; page numbers outside the pool count as `bad`.
__device__ __forceinline__ long long kv_row(const KvArgs &a, int layer, int page, int head, int off)
{
    return (((((long long)layer * a.num_pages + page) * a.heads + head) << a.page_shift) + off);
}

// ---- division of the attention's work -----------------------------------------------------------
// An ITEM is a tile of rows of one sequence and key/value head (row r of a chunk is head r % group of token r / group);
// its cost is the number of UNITS of positions that its rows see (at least one, so that every row is written).  How many
// rows and positions that is, a kernel's Shape says.  A WORKER is a CTA, or a cluster of CTAs that split every unit among
// them and join their results through shared memory.  Worker i of n gets
//
//   few items: a piece of ONE item.  Every item is cut into pieces of at most L units, L the least for which there are
//       workers for all pieces, if that is within an eighth and four units of an even share W / n: nobody starts a second
//       item, whose fixed cost (queries, join) is several units.
//   otherwise: units i W / n .. (i + 1) W / n - 1 of all W units in the order (sequence, row tile, head), so that the
//       workers finish together however ragged the batch is; a worker has the tail of one item, some whole items and
//       the head of another.
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
    static __device__ __forceinline__ int units(const AttendArgs &a, const Chunk &k, int r)
    {
        int seen = k.total;
        if (!a.mask) seen = min(seen, k.ctx + min(k.len - 1, a.by_group.div((r + 1) * (int)a.by_rows.d - 1)) + 1);
        return max(1, a.by_unit.ceil(seen));
    }
};

template <typename Shape>
struct KvPlan {
    long long W, hi, u;         // many items: units in all; end of this worker's; next unit
    int n;                      // workers (0: a piece each)
    int b, rt, head, kt;        // item of unit u, and its place there
    int pieces, piece;          // of the item, and this worker's
    int c0;
    bool first;
    Chunk c;

    // Pieces of at most L units of one head of sequence bb (L = 1: its units).  One copy of this code serves every pass
    // below: a kernel starts with a cold instruction cache, where straight-line copies cost more than the arithmetic.
    static __device__ __noinline__ unsigned pieces_of(const AttendArgs &a, int bb, unsigned L, unsigned *items)
    {
        const Chunk k = kv_chunk(a.kv, bb);
        const int nr = Shape::row_tiles(a, k);
        unsigned p = 0;
#pragma unroll 1
        for (int r = 0; r < nr; ++r) {
            const unsigned u = Shape::units(a, k, r);
            p += L == 1 ? u : (u + L - 1) / L;
        }
        *items = nr;
        return p;
    }
    // Sum over the sequences of pieces_of, or (find >= 0) the sequence that piece `find` belongs to and the pieces before it.
    static __device__ __noinline__ long long scan(const AttendArgs &a, int lane, unsigned L, long long find, int *b, long long *out)
    {
        long long before = 0, items = 0;
#pragma unroll 1
        for (int b0 = 0; b0 < a.kv.B; b0 += 32) {
            unsigned n = 0;
            const long long own = b0 + lane < a.kv.B ? (long long)pieces_of(a, b0 + lane, L, &n) * a.kv.heads : 0;
            long long incl = own;
            items += n;
#pragma unroll 1
            for (int o = 1; o < 32; o <<= 1) {
                const long long x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                if (lane >= o) incl += x;
            }
            const unsigned m = find >= 0 ? __ballot_sync(0xFFFFFFFFu, before + incl > find) : 0;
            if (m) {
                const int l = __ffs(m) - 1;
                *b = b0 + l;
                *out = before + __shfl_sync(0xFFFFFFFFu, incl - own, l);
                return 1;
            }
            before += __shfl_sync(0xFFFFFFFFu, incl, 31);
        }
        if (find >= 0) return 0;
#pragma unroll 1
        for (int o = 16; o > 0; o >>= 1) items += __shfl_xor_sync(0xFFFFFFFFu, items, o);
        *out = items * a.kv.heads;
        return before;
    }

    // Called by all 32 lanes of a warp of worker `me` of `count`; false = nothing to do.  No piece is
    // smaller than `least` units unless its item is.
    __device__ bool start(const AttendArgs &a, int lane, int me, int count, int least)
    {
        long long items, before;
        W = scan(a, lane, 1, -1, &b, &items);
        first = true;
        if (W == 0) return false;
        n = (int)min((long long)count, (W + least - 1) / least);
        const long long even = max((W + count - 1) / count, (long long)least), most = even + even / 8 + 4;
        unsigned L = 1;
        long long find;
        bool each = false;
#pragma unroll 1
        for (long long LL = even; items <= count && LL <= most && !each; LL += (LL + 15) / 16) {
            long long ignored;
            L = (unsigned)LL;
            each = scan(a, lane, L, -1, &b, &ignored) <= count;
        }
        if (each) {
            n = 0;
            find = me;
        } else {
            if (me >= n) return false;
            L = 1;
            find = u = W * me / n;
            hi = W * (me + 1) / n;
        }
        if (!scan(a, lane, L, find, &b, &before)) return false;
        c = kv_chunk(a.kv, b);
        long long rest = find - before;
#pragma unroll 1
        for (rt = 0;; ++rt) {
            pieces = (int)(((unsigned)Shape::units(a, c, rt) + L - 1) / L);
            const long long t = (long long)pieces * a.kv.heads;
            if (rest < t) break;
            rest -= t;
        }
        head = (int)(rest / pieces);
        kt = piece = (int)(rest % pieces);
        c0 = me - piece;
        return true;
    }
    __device__ __forceinline__ int owner(long long t) const { return (int)(((t + 1) * n - 1) / W); }

    // The next segment; false when the worker has done its share.  Uniform over the worker.
    __device__ bool next(const AttendArgs &a, Segment &s)
    {
        if (n == 0 ? !first : u >= hi) return false;
        const int units = Shape::units(a, c, rt);
        s.b = b;
        s.rt = rt;
        s.head = head;
        s.slot = first ? 0 : 1;
        first = false;
        if (n == 0) {
            s.kt0 = (int)((long long)units * piece / pieces);
            s.kt1 = (int)((long long)units * (piece + 1) / pieces);
            s.c0 = c0;
            s.c1 = c0 + pieces - 1;
            s.slot0 = 0;
            return true;
        }
        s.kt0 = kt;
        s.kt1 = (int)min((long long)units, kt + (hi - u));
        const long long item = u - kt;
        s.c0 = owner(item);
        s.c1 = owner(item + units - 1);
        s.slot0 = W * s.c0 / n == item ? 0 : 1;
        u += s.kt1 - s.kt0;
        kt = s.kt1;
        return true;
    }
    // Moves on to the next item (call after the segment's work, when its chunk is no longer needed).
    __device__ void advance(const AttendArgs &a)
    {
        if (n == 0 || u >= hi || kt < Shape::units(a, c, rt)) return;
        kt = 0;
        if (++head < a.kv.heads) return;
        head = 0;
        if (++rt < Shape::row_tiles(a, c)) return;
        rt = 0;
        do {
            ++b;
            c = kv_chunk(a.kv, b);
        } while (c.len == 0);            // ends: u < hi means that a later sequence has units
    }
};

}  // namespace dresd
