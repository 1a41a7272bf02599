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
    static constexpr float kBound = 61440.f;             // 240 x 2^8: the largest value that is finite after rounding
};
template <> struct KvType<__nv_bfloat16> {
    static constexpr int kMinExp = -126;
    static constexpr float kBound = 3.1901471898837980e38f;   // 1.875 x 2^127
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
// rows and positions that is, a kernel's Shape says.  The items in the order (sequence, row tile, head) form one
// line of W units, and CTA i of n takes units i W / n .. (i + 1) W / n - 1 of it, whatever the
// lengths: the CTAs finish together however ragged the batch is.  A CTA therefore works on the tail
// of one item, some whole items and the head of another.  Parts of an item are joined by the CTA that
// finishes it last, in the order of the CTAs, so results do not depend on timing.
struct Segment {
    int b, rt, head;        // the item
    int kt0, kt1;           // its units that this CTA takes
    int n_kt;               // its units in all
    int c0, c1;             // CTAs that share it
    int slot;               // slot of this CTA's part (0: it is the CTA's first segment, 1: a later one)
    int slot0;              // slot of c0's part; those of c0 + 1 .. c1 are 0
};

// Shape of the kernel for few rows: tiles of kRows rows, units of kTile positions.
template <int kRows, int kTile>
struct FewRows {
    static __device__ __forceinline__ int row_tiles(const AttendArgs &a, const Chunk &k) { return (k.len * a.group + kRows - 1) / kRows; }
    static __device__ __forceinline__ int units(const AttendArgs &a, const Chunk &k, int r)
    {
        int seen = k.total;
        if (!a.mask) seen = min(seen, k.ctx + min(k.len - 1, ((r + 1) * kRows - 1) / a.group) + 1);
        return max(1, (seen + kTile - 1) / kTile);
    }
};

template <typename Shape>
struct KvPlan {
    long long W, hi, u;         // units in all; end of this CTA's; next unit
    int n, cta;
    int b, rt, head, kt;        // item of unit u, and its place there
    bool first;
    Chunk c;

    static __device__ __forceinline__ long long cost(const AttendArgs &a, int bb)
    {
        const Chunk k = kv_chunk(a.kv, bb);
        const int nr = Shape::row_tiles(a, k);
        long long t = 0;
        for (int r = 0; r < nr; ++r) t += Shape::units(a, k, r);
        return t * a.kv.heads;
    }

    // Called by all 32 lanes of a warp; false = nothing to do.  Small problems are not spread over more
    // CTAs than give each `least` units.
    __device__ bool start(const AttendArgs &a, int lane, int least)
    {
        const int B = a.kv.B;
        cta = blockIdx.x;
        long long mine = 0;
        for (int b0 = 0; b0 < B; b0 += 32) mine += b0 + lane < B ? cost(a, b0 + lane) : 0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xFFFFFFFFu, mine, o);
        W = mine;
        n = (int)min((long long)gridDim.x, (W + least - 1) / least);
        if (cta >= n) return false;
        const long long lo = u = W * cta / n;
        hi = W * (cta + 1) / n;
        // the sequence that unit `lo` belongs to
        long long before = 0;
        b = 0;
        for (int b0 = 0; b0 < B; b0 += 32) {
            const long long own = b0 + lane < B ? cost(a, b0 + lane) : 0;
            long long incl = own;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                if (lane >= o) incl += x;
            }
            const unsigned m = __ballot_sync(0xFFFFFFFFu, before + incl > lo);
            if (m) {
                const int l = __ffs(m) - 1;
                b = b0 + l;
                before += __shfl_sync(0xFFFFFFFFu, incl - own, l);
                break;
            }
            before += __shfl_sync(0xFFFFFFFFu, incl, 31);
        }
        c = kv_chunk(a.kv, b);
        long long rest = lo - before;
        for (rt = 0;; ++rt) {
            const long long t = (long long)Shape::units(a, c, rt) * a.kv.heads;
            if (rest < t) break;
            rest -= t;
        }
        const int nk = Shape::units(a, c, rt);
        head = (int)(rest / nk);
        kt = (int)(rest % nk);
        first = true;
        return true;
    }
    __device__ __forceinline__ int owner(long long t) const { return (int)(((t + 1) * n - 1) / W); }

    // The next segment; false when the CTA has done its share.  Uniform over the CTA.
    __device__ bool next(const AttendArgs &a, Segment &s)
    {
        if (u >= hi) return false;
        s.n_kt = Shape::units(a, c, rt);
        s.b = b;
        s.rt = rt;
        s.head = head;
        s.kt0 = kt;
        s.kt1 = (int)min((long long)s.n_kt, kt + (hi - u));
        const long long item = u - kt;
        s.c0 = owner(item);
        s.c1 = owner(item + s.n_kt - 1);
        s.slot = first ? 0 : 1;
        s.slot0 = W * s.c0 / n == item ? 0 : 1;
        first = false;
        u += s.kt1 - s.kt0;
        kt = s.kt1;
        return true;
    }
    // Moves on to the next item (call after the segment's work, when its chunk is no longer needed).
    __device__ void advance(const AttendArgs &a)
    {
        if (u >= hi || kt < Shape::units(a, c, rt)) return;
        kt = 0;
        if (++head < a.kv.heads) return;
        head = 0;
        if (++rt < Shape::row_tiles(a, c)) return;
        rt = 0;
        do {
            ++b;
            c = kv_chunk(a.kv, b);
        } while (c.len == 0);            // ends: u < hi means that a later sequence has tiles
    }
};

}  // namespace dresd
