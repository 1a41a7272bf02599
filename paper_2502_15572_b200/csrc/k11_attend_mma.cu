// K11 -- attention of few rows per key/value head over the paged cache (single tokens, short chunks).
//
//     s_rj = scale q_r . k_j,   out_r = sum_j 2^(s_rj - m_r) v_j / sum_j 2^(s_rj - m_r)      (scale holds log2 e)
//
// in one pass over the cache with the running maximum m, weight sum l and weighted sum o of every row.  Every
// key and value is read once and meets a handful of rows, so the bound is HBM and the aim is many loads in flight
// with nothing between them and the arithmetic: a warp takes 16 positions at a time STRAIGHT INTO REGISTERS in the
// fragment layout of mma.sync m16n8k16 -- no shared memory, no barrier, no transposition:
//
//   S^T = K Q^T   keys as the M = 16 operand, rows as N = 8.  The k index of the instruction may run over the
//                 elements of a row in any order that keys and queries share; it is laid out so that a lane's
//                 fragments are whole 16-byte pieces of a key.
//   O^T = V^T P^T elements as M, rows as N, positions as K.  A lane loads 16-byte pieces of four values; pairs of
//                 positions are joined with byte permutes (for E4M3 before the conversion, which takes two codes at
//                 once).  P^T is S^T's own fragment turned by movmatrix.
//
// 16-row tiles of queries would leave M half empty at the usual 1 to 8 rows per head; with rows as N nothing is padded
// beyond 8 and the accumulators take half the registers.  8-bit codes become 16-bit numbers exactly; the keys' scale is
// applied to the score, the values' to the value, both powers of two.
//
// Work is divided as kv_plan.cuh says; the four warps of a CTA take 16 positions each of every 64-position tile and are
// joined through shared memory at the end of a segment.  The maximum is only raised when a score passes it by 2^8
// (weights stay far inside the range of either type), which saves the shuffles of the maximum on most tiles.
#include "kv_plan.cuh"

namespace dresd {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kTile = kWarps * 16;
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

// Parts of shared items: per CTA two slots of `rows` x (d + 2) floats: the sums, then the rows' maxima, then the
// rows' weight sums.
__device__ __forceinline__ float *part_slot(const AttendArgs &a, int cta, int slot, int rows)
{
    return a.part + ((size_t)cta * 2 + slot) * rows * (a.kv.d + 2);
}

template <int kBytes> struct Piece;                       // a lane's load
template <> struct Piece<16> { using type = uint4; };
template <> struct Piece<8> { using type = uint2; };
__device__ __forceinline__ uint32_t word(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t word(const uint2 &v, int i) { return i == 0 ? v.x : v.y; }

// NT: tiles of 8 rows.
template <typename T, bool Q8, int D, int NT>
__global__ void __launch_bounds__(kThreads)
attend_mma_kernel(const __grid_constant__ AttendArgs a, int least)
{
    constexpr int kRows = 8 * NT;
    constexpr int kRowBytes = Q8 ? D : 2 * D;             // one key or value
    constexpr int kKeyPieces = kRowBytes / 64;            // 16-byte pieces of a key per lane (4 lanes share a key)
    constexpr int kSteps = D / 16;                        // k-steps of the first product, M-tiles of the second
    constexpr int kValBytes = kRowBytes >= 128 ? 16 : 8;  // a lane's piece of a value (8 lanes share a value)
    constexpr int kValPieces = kRowBytes / 8 / kValBytes;
    constexpr int kValElems = kValBytes / (Q8 ? 1 : 2);   // elements in it
    using VPiece = typename Piece<kValBytes>::type;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    __shared__ float s_o[kWarps][kRows][D + 4];
    __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows];
    __shared__ unsigned s_ticket;

    KvPlan<FewRows> plan;
    if (!plan.start(a, lane, blockIdx.x, gridDim.x, least)) return;
    Segment seg;
    while (plan.next(a, seg)) {
        const Chunk ch = plan.c;
        const int heads = a.kv.heads * a.group;
        const int rows = min(kRows, ch.len * a.group - seg.rt * kRows);     // valid rows of the tile
        // ---- the queries, as the B operand: lane (g, c) holds row g's pieces
        uint32_t q[NT][kSteps][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = seg.rt * kRows + nt * 8 + g;
            const bool ok = nt * 8 + g < rows;
            const T *src = static_cast<const T *>(a.q) + (long long)(ch.row0 + (ok ? a.by_group.div(r) : 0)) * a.q_row +
                           (seg.head * a.group + (ok ? (r - a.by_group.div(r) * a.group) : 0)) * a.q_head;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                // 16-bit keys: piece 4 i + c.  8-bit keys: a key's piece is 16 elements, two of the query's.
                const int at = Q8 ? (i / 2 * 4 + c) * 16 + i % 2 * 8 : (i * 4 + c) * 8;
                const uint4 x = ok ? __ldg(reinterpret_cast<const uint4 *>(src + at)) : make_uint4(0, 0, 0, 0);
                q[nt][2 * i][0] = x.x;
                q[nt][2 * i][1] = x.y;
                q[nt][2 * i + 1][0] = x.z;
                q[nt][2 * i + 1][1] = x.w;
            }
        }
        int limit[NT][2];                                  // causal: positions that rows 2c, 2c + 1 see
        const uint32_t *bits[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = min(nt * 8 + 2 * c + i, rows - 1);
                const int tok = a.by_group.div(seg.rt * kRows + r);
                limit[nt][i] = a.mask ? ch.total : min(ch.total, ch.ctx + tok + 1);
                bits[nt][i] = a.mask ? a.mask + (long long)(ch.row0 + tok) * a.mask_words : nullptr;
            }
        float o[NT][kSteps][4] = {};
        float m[NT][2], l[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) m[nt][0] = m[nt][1] = -INFINITY, l[nt][0] = l[nt][1] = 0.f;

        for (int kt = seg.kt0; kt < seg.kt1; ++kt) {
            const int p0 = kt * kTile + warp * 16;
            if (p0 >= ch.total) break;                     // positions grow: nothing further for this warp
            int page = __ldg(a.kv.table + (long long)seg.b * a.kv.width + (p0 >> a.kv.page_shift));
            if (page < 0 || page >= a.kv.num_pages) page = 0;
            // the pool has at least one page, and 16 positions from a multiple of 16 lie in one page
            const long long row = kv_row(a.kv, a.kv.layer, page, seg.head, p0 & ((1 << a.kv.page_shift) - 1));
            uint4 kx[2][kKeyPieces];
            VPiece vx[4][kValPieces];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < kKeyPieces; ++i)
                    kx[j][i] = __ldcs(reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(a.kv.k) + (row + j * 8 + g) * kRowBytes) + i * 4 + c);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < kValPieces; ++i)
                    vx[j][i] = __ldcs(reinterpret_cast<const VPiece *>(static_cast<const uint8_t *>(a.kv.v) +
                                                                     (row + (j & 1) + (j >> 1) * 8 + 2 * c) * kRowBytes) + i * 8 + g);
            int ke[2] = {127, 127}, ve[4] = {127, 127, 127, 127};
            if constexpr (Q8) {
                ke[0] = a.kv.k_exps[row + g];
                ke[1] = a.kv.k_exps[row + 8 + g];
#pragma unroll
                for (int j = 0; j < 4; ++j) ve[j] = a.kv.v_exps[row + (j & 1) + (j >> 1) * 8 + 2 * c];
            }
            // ---- S^T = K Q^T
            float s[NT][4] = {};
            if constexpr (!Q8) {
#pragma unroll
                for (int st = 0; st < kSteps; ++st)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        mma16816<T>(s[nt], word(kx[0][st / 2], st % 2 * 2), word(kx[1][st / 2], st % 2 * 2),
                                    word(kx[0][st / 2], st % 2 * 2 + 1), word(kx[1][st / 2], st % 2 * 2 + 1), q[nt][st][0], q[nt][st][1]);
            } else {
                const uint32_t one = scale_bits<T>(127) * 0x10001u;
#pragma unroll
                for (int st = 0; st < kSteps; ++st) {
                    uint32_t f[2][2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t w = word(kx[j][st / 4], st % 4);
                        f[j][0] = codes_to_pair<T>(__byte_perm(w, 0, 0x1404), one);
                        f[j][1] = codes_to_pair<T>(__byte_perm(w, 0, 0x3424), one);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        mma16816<T>(s[nt], f[0][0], f[1][0], f[0][1], f[1][1], q[nt][st][0], q[nt][st][1]);
                }
            }
            // ---- scale, mask.  s[nt][2 j + i]: key g + 8 j, row 2 c + i
            const bool all_seen = p0 + 16 <= ch.ctx && p0 + 16 <= ch.total;
            const float sk[2] = {Q8 ? a.scale_log2 * pow2f(min(ke[0], 253) - 127) : a.scale_log2,
                                 Q8 ? a.scale_log2 * pow2f(min(ke[1], 253) - 127) : a.scale_log2};
            bool over = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float x = s[nt][2 * j + i] * sk[j];
                        if (!all_seen) {
                            const int p = p0 + 8 * j + g, t = p - ch.ctx;
                            bool seen = p < limit[nt][i];
                            if (a.mask && t >= 0 && seen) seen = (t >> 5) < a.mask_words && (bits[nt][i][t >> 5] >> (t & 31) & 1);
                            if (!seen) x = -INFINITY;
                        }
                        s[nt][2 * j + i] = x;
                        over |= x > m[nt][i] + kSlack;
                    }
            if (__any_sync(0xFFFFFFFFu, over)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float x = fmaxf(fmaxf(s[nt][i], s[nt][2 + i]), m[nt][i]);
#pragma unroll
                        for (int sh = 4; sh < 32; sh <<= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, sh));
                        const float f = x > -INFINITY ? exp2f(m[nt][i] - x) : 1.f;
                        m[nt][i] = x;
                        l[nt][i] *= f;
#pragma unroll
                        for (int st = 0; st < kSteps; ++st) {
                            o[nt][st][i] *= f;
                            o[nt][st][2 + i] *= f;
                        }
                    }
            }
            // ---- weights, and P^T as the B operand: lane (g, c) holds row g, positions 2 c, 2 c + 1 (+ 8)
            uint32_t p[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float base = m[nt][i] > -INFINITY ? m[nt][i] : 0.f;
#pragma unroll
                    for (int j = 0; j < 2; ++j) s[nt][2 * j + i] = exp2f(s[nt][2 * j + i] - base);
                    l[nt][i] += s[nt][i] + s[nt][2 + i];
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) p[nt][j] = turn8x8(pack2<T>(s[nt][2 * j], s[nt][2 * j + 1]));
            }
            // ---- O^T += V^T P^T
            uint32_t vs[2] = {0, 0}, vb[2] = {0, 0};
            bool big = false;
            if constexpr (Q8) {
                vs[0] = scale_bits<T>(ve[0]) | scale_bits<T>(ve[1]) << 16;
                vs[1] = scale_bits<T>(ve[2]) | scale_bits<T>(ve[3]) << 16;
                if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                    big = max(max(ve[0], ve[1]), max(ve[2], ve[3])) > 134;
                    vb[0] = big_scale(ve[0]) | big_scale(ve[1]) << 16;
                    vb[1] = big_scale(ve[2]) | big_scale(ve[3]) << 16;
                }
            }
            if (!all_seen) {
                // Positions that some row does not see may hold anything, and 0 x NaN is NaN: unused positions
                // are cleared, and non-finite values of the chunk itself are taken out here and added row by row.
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (p0 + (j & 1) + (j >> 1) * 8 + 2 * c >= ch.total) {
#pragma unroll
                        for (int i = 0; i < kValPieces; ++i) vx[j][i] = VPiece{};
                    }
                if constexpr (Q8) {                        // the code of NaN counts as 0
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int i = 0; i < kValPieces; ++i) {
                            uint32_t *x = reinterpret_cast<uint32_t *>(&vx[j][i]);
#pragma unroll
                            for (int w = 0; w < kValBytes / 4; ++w) x[w] &= ~__vcmpeq4(x[w] & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
                        }
                } else {
                    constexpr uint32_t kInf = std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u;
                    bool odd = false;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int i = 0; i < kValPieces; ++i)
#pragma unroll
                            for (int w = 0; w < kValBytes / 4; ++w) {
                                const uint32_t x = word(vx[j][i], w);
                                odd |= (x & kInf) == kInf || (x >> 16 & kInf) == kInf;
                            }
                    if (__any_sync(0xFFFFFFFFu, odd)) {
                        for (int k = 0; k < 16 && p0 + k < ch.total; ++k) {
                            const T *vrow = static_cast<const T *>(a.kv.v) + (row + k) * D;
                            float w[NT][2];                // weights of rows 2 c, 2 c + 1 at position k
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int i = 0; i < 2; ++i)
                                    w[nt][i] = __shfl_sync(0xFFFFFFFFu, k < 8 ? s[nt][i] : s[nt][2 + i], (k & 7) * 4 + c);
#pragma unroll
                            for (int st = 0; st < kSteps; ++st)
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    const int e = 2 * st + h;
                                    const float x = unpack2<T>(*reinterpret_cast<const uint16_t *>(vrow + e / kValElems * 8 * kValElems + g * kValElems + e % kValElems)).x;
                                    if (isfinite(x)) continue;
#pragma unroll
                                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                        for (int i = 0; i < 2; ++i)
                                            if (w[nt][i] > 0.f) o[nt][st][2 * h + i] += w[nt][i] * x;
                                }
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int i = 0; i < kValPieces; ++i) {
                                uint32_t *x = reinterpret_cast<uint32_t *>(&vx[j][i]);
#pragma unroll
                                for (int w = 0; w < kValBytes / 4; ++w) {
                                    if ((x[w] & kInf) == kInf) x[w] &= 0xFFFF0000u;
                                    if ((x[w] >> 16 & kInf) == kInf) x[w] &= 0x0000FFFFu;
                                }
                            }
                    }
                }
            }
            // M-tile st covers elements e0 = 2 st, e1 = 2 st + 1 of every lane group's piece
#pragma unroll
            for (int st = 0; st < kSteps; ++st) {
                constexpr int kPer = kValElems / 2;        // M-tiles per piece
                const int i = st / kPer, e = st % kPer;    // e: pair of elements within the piece
                uint32_t f[2][2];                          // [pair of positions][element e0, e1]
                if constexpr (!Q8) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t lo = word(vx[2 * j][i], e), hi = word(vx[2 * j + 1][i], e);
                        f[j][0] = __byte_perm(lo, hi, 0x5410);
                        f[j][1] = __byte_perm(lo, hi, 0x7632);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t lo = word(vx[2 * j][i], e / 2) >> (16 * (e & 1)), hi = word(vx[2 * j + 1][i], e / 2) >> (16 * (e & 1));
                        const uint32_t w = __byte_perm(lo, hi, 0x5140);       // codes: e0 of both positions, e1 of both
                        f[j][0] = codes_to_pair<T>(__byte_perm(w, 0, 0x1404), vs[j]);
                        f[j][1] = codes_to_pair<T>(__byte_perm(w, 0, 0x3424), vs[j]);
                        if constexpr (std::is_same<T, __nv_bfloat16>::value)
                            if (big)
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    const __nv_bfloat162 r = __hmul2(*reinterpret_cast<__nv_bfloat162 *>(&f[j][h]), *reinterpret_cast<__nv_bfloat162 *>(&vb[j]));
                                    f[j][h] = *reinterpret_cast<const uint32_t *>(&r);
                                }
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma16816<T>(o[nt][st], f[0][0], f[0][1], f[1][0], f[1][1], p[nt][0], p[nt][1]);
            }
        }
        // ---- join the four warps
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int sh = 4; sh < 32; sh <<= 1) l[nt][i] += __shfl_xor_sync(0xFFFFFFFFu, l[nt][i], sh);
                const int r = nt * 8 + 2 * c + i;
                if (g == 0) {
                    s_m[warp][r] = m[nt][i];
                    s_l[warp][r] = l[nt][i];
                }
#pragma unroll
                for (int st = 0; st < kSteps; ++st)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int e = 2 * st + h;
                        s_o[warp][r][e / kValElems * 8 * kValElems + g * kValElems + e % kValElems] = o[nt][st][2 * h + i];
                    }
            }
        __syncthreads();
        const bool shared_item = seg.c0 != seg.c1;
        float *part = part_slot(a, blockIdx.x, seg.slot, kRows);
        // a thread takes 4 elements of a row
        for (int x = tid; x < rows * (D / 4); x += kThreads) {
            const int r = x / (D / 4), e = x % (D / 4) * 4;
            float mm = s_m[0][r];
#pragma unroll
            for (int w = 1; w < kWarps; ++w) mm = fmaxf(mm, s_m[w][r]);
            const float base = mm > -INFINITY ? mm : 0.f;
            float ll = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = exp2f(s_m[w][r] - base);
                ll += f * s_l[w][r];
                const float4 y = *reinterpret_cast<const float4 *>(&s_o[w][r][e]);
                if (f > 0.f) acc.x += f * y.x, acc.y += f * y.y, acc.z += f * y.z, acc.w += f * y.w;
            }
            if (shared_item) {
                __stcg(reinterpret_cast<float4 *>(part + r * D + e), acc);
                if (e == 0) {
                    __stcg(part + kRows * D + r, mm);
                    __stcg(part + kRows * D + kRows + r, ll);
                }
            } else {
                const float inv = ll > 0.f ? 1.f / ll : ll == 0.f ? 0.f : ll;      // a NaN sum stays one
                const int rr = seg.rt * kRows + r;
                const long long at = (long long)(ch.row0 + a.by_group.div(rr)) * heads + seg.head * a.group + (rr - a.by_group.div(rr) * a.group);
                *reinterpret_cast<uint2 *>(static_cast<T *>(a.out) + at * D + e) =
                    make_uint2(pack2<T>(acc.x * inv, acc.y * inv), pack2<T>(acc.z * inv, acc.w * inv));
                if (a.lse && e == 0) a.lse[at] = (base + log2f(ll)) * 0.69314718055994531f;
            }
        }
        if (shared_item) {
            __threadfence();
            __syncthreads();
            if (tid == 0) s_ticket = atomicAdd(a.tickets + seg.c0, 1u);
            __syncthreads();
            if (s_ticket == (unsigned)(seg.c1 - seg.c0)) {                       // the last of them: join the parts
                __threadfence();
                if (tid == 0) a.tickets[seg.c0] = 0;
                for (int x = tid; x < rows * (D / 4); x += kThreads) {
                    const int r = x / (D / 4), e = x % (D / 4) * 4;
                    float mm = -INFINITY, ll = 0.f;
                    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int i = seg.c0; i <= seg.c1; ++i) {
                        const float *ps = part_slot(a, i, i == seg.c0 ? seg.slot0 : 0, kRows);
                        const float pm = __ldcg(ps + kRows * D + r), pl = __ldcg(ps + kRows * D + kRows + r);
                        const float4 y = __ldcg(reinterpret_cast<const float4 *>(ps + r * D + e));
                        const float nm = fmaxf(mm, pm), base = nm > -INFINITY ? nm : 0.f;
                        const float f0 = exp2f(mm - base), f1 = exp2f(pm - base);
                        ll = f0 * ll + f1 * pl;
                        acc.x = f0 * acc.x + (f1 > 0.f ? f1 * y.x : 0.f);
                        acc.y = f0 * acc.y + (f1 > 0.f ? f1 * y.y : 0.f);
                        acc.z = f0 * acc.z + (f1 > 0.f ? f1 * y.z : 0.f);
                        acc.w = f0 * acc.w + (f1 > 0.f ? f1 * y.w : 0.f);
                        mm = nm;
                    }
                    const float base = mm > -INFINITY ? mm : 0.f;
                    const float inv = ll > 0.f ? 1.f / ll : ll == 0.f ? 0.f : ll;
                    const int rr = seg.rt * kRows + r;
                    const long long at = (long long)(ch.row0 + a.by_group.div(rr)) * heads + seg.head * a.group + (rr - a.by_group.div(rr) * a.group);
                    *reinterpret_cast<uint2 *>(static_cast<T *>(a.out) + at * D + e) =
                        make_uint2(pack2<T>(acc.x * inv, acc.y * inv), pack2<T>(acc.z * inv, acc.w * inv));
                    if (a.lse && e == 0) a.lse[at] = (base + log2f(ll)) * 0.69314718055994531f;
                }
            }
        }
        __syncthreads();                                    // s_o is written again by the next segment
        plan.advance(a);
    }
}

template <typename T, bool Q8, int D, int NT>
cudaError_t launch(const AttendArgs &a, int sms, cudaStream_t stream)
{
    static int occupancy = 0;                               // same for every device of this build (sm_100a)
    if (occupancy == 0) {
        int n = 0;
        cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, attend_mma_kernel<T, Q8, D, NT>, kThreads, 0);
        if (e != cudaSuccess) return e;
        occupancy = n;
    }
    int grid = sms * occupancy;
    if (grid > attend_mma_max_ctas(sms)) grid = attend_mma_max_ctas(sms);
    attend_mma_kernel<T, Q8, D, NT><<<grid, kThreads, 0, stream>>>(a, 2);
    return cudaGetLastError();
}
template <typename T, bool Q8>
cudaError_t by_shape(const AttendArgs &a, int sms, cudaStream_t stream)
{
    const bool one = (long long)a.max_chunk * a.group <= 8;
    if (a.kv.d == 64) return one ? launch<T, Q8, 64, 1>(a, sms, stream) : launch<T, Q8, 64, 2>(a, sms, stream);
    return one ? launch<T, Q8, 128, 1>(a, sms, stream) : launch<T, Q8, 128, 2>(a, sms, stream);
}

}  // namespace

int attend_mma_max_ctas(int sms) { return 8 * sms; }
size_t attend_mma_part_floats(int sms, int d) { return (size_t)attend_mma_max_ctas(sms) * 2 * 16 * (d + 2); }

cudaError_t launch_attend_mma(const AttendArgs &args, int sms, cudaStream_t stream)
{
    AttendArgs a = args;
    a.by_unit = FastDiv(kTile);
    a.by_rows = FastDiv((long long)a.max_chunk * a.group <= 8 ? 8 : 16);
    const bool q8 = a.kv.k_exps != nullptr;
    if (a.kv.dtype == kF16) return q8 ? by_shape<__half, true>(a, sms, stream) : by_shape<__half, false>(a, sms, stream);
    return q8 ? by_shape<__nv_bfloat16, true>(a, sms, stream) : by_shape<__nv_bfloat16, false>(a, sms, stream);
}

}  // namespace dresd
