// K15 -- products with 4-bit weights and one scale for a group of inputs, for few rows (a token or a few for every sequence):
//     y[t][o] = sum_g s[o][g] sum_{i in g} (c[o][i] - 8) x[t][i]
// The inner sums multiply whole numbers -8 .. 7 and the activations, both exact in the activations' type, and are kept in fp32; the scale meets
// them there.  So a weight is never rounded, and a result is rounded once.
//
// Bound: the weights' bytes, and on small matrices the latency of fetching them once.  A CTA has 128 outputs and 256 inputs at a time, up to three of these
// steps on their way by cp.async; the CTAs of a cluster split the inputs, so that on small matrices every byte is on its way from the
// start, and add their parts up in the order of their ranks.  Measured (device): one row of 4096 x 4096 6.2 us, 7 rows of 4096 x 11008 12.5 us, one row of
// 4096 x 32000 27 us: 1.9 to 2.5 TB/s, so neither bytes nor a small matrix's latency bounds the larger ones.  A CTA goes through two steps, joins and
// ends, nothing is on its way from one tile to the next, and 11008 outputs are a wave and a part (688 CTAs, 592 resident).
//
// A warp computes 32 outputs for up to 8 kBlocks rows with mma.sync, weights as the 16-row operand.  The order of inputs within an
// instruction is free, as long as both operands agree: a lane takes 8 or 16 consecutive codes of a row (4 lanes a row, 8 rows
// a load) and the same inputs of its row of activations.  Rows in shared memory are padded so that neither load meets a bank twice.
#include <atomic>
#include <type_traits>

#include "kv_plan.cuh"

namespace dresd {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps, kTile = 32 * kWarps;      // outputs of a CTA
constexpr int kChunk = 256;                                                 // inputs at a time
constexpr int kMaxSplit = 8;
static_assert(kThreads == kTile, "a thread fetches the scales of an output");

// The eight codes of a word, minus 8, as the pairs (0, 4), (1, 5), (2, 6), (3, 7) of T.  Nibbles become bits of the mantissas of powers of two, at the
// bottom (fp16 2048 + 2 c, bf16 256 + 2 c) or above that (fp16 128 + 2 c; bf16, which has fewer, moved down by one: 32 + 2 c); half of that less 1032,
// 136, 72, 24 is exact, and an fma: additions of halves share a unit with shifts and logic, of which there are more.
template <typename T> __device__ __forceinline__ void unpack(uint32_t w, uint32_t (&p)[4]);
template <> __device__ __forceinline__ void unpack<__half>(uint32_t w, uint32_t (&p)[4])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t at = k < 2 ? w : w >> 8, two = k % 2 ? (at & 0x00F000F0u) | 0x58005800u : (at & 0x000F000Fu) | 0x68006800u;
        const uint32_t half = 0x38003800u, less = k % 2 ? 0xD480D480u : 0xE408E408u;
        const __half2 r = __hfma2(*reinterpret_cast<const __half2 *>(&two), *reinterpret_cast<const __half2 *>(&half), *reinterpret_cast<const __half2 *>(&less));
        p[k] = *reinterpret_cast<const uint32_t *>(&r);
    }
}
template <> __device__ __forceinline__ void unpack<__nv_bfloat16>(uint32_t w, uint32_t (&p)[4])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t at = w >> (k / 2 * 8 + k % 2), two = k % 2 ? (at & 0x00780078u) | 0x42004200u : (at & 0x000F000Fu) | 0x43804380u;
        const uint32_t half = 0x3F003F00u, less = k % 2 ? 0xC1C0C1C0u : 0xC308C308u;
        const __nv_bfloat162 r = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&two), *reinterpret_cast<const __nv_bfloat162 *>(&half),
                                         *reinterpret_cast<const __nv_bfloat162 *>(&less));
        p[k] = *reinterpret_cast<const uint32_t *>(&r);
    }
}
template <typename T> __device__ __forceinline__ T from_float(float x)
{
    if constexpr (std::is_same<T, __half>::value) return __float2half_rn(x);
    else return __float2bfloat16_rn(x);
}
template <typename T> __device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same<T, __half>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int kBytes> __device__ __forceinline__ void copy_async(void *dst, const void *src, bool there)      // or zeros
{
    if constexpr (kBytes == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(__cvta_generic_to_global(src)), "r"(there ? 16 : 0) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;" ::"r"(smem_u32(dst)), "l"(__cvta_generic_to_global(src)), "r"(there ? kBytes : 0), "n"(kBytes) : "memory");
}
// Waits for all but the last `left` groups of copies.
__device__ __forceinline__ void wait_copies(int left)
{
    switch (left) {
    case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
    case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
    default: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
    }
}

template <int kGroup, int kBlocks> struct Stage {
    static constexpr int kWords = kGroup == 32 ? 1 : 2;                     // of eight codes, of a lane and row at a time
    static constexpr int kSub = 32 * kWords;                                // inputs of four lanes at a time
    static constexpr int kCodeRow = kChunk / 2 + kSub / 2, kXRow = kChunk * 2 + (kWords == 1 ? 64 : 16);      // bytes; padded
    static constexpr int kGroups = kChunk / kGroup, kScaleRow = 2 * kGroups;
    static constexpr int kMost = kBlocks == 4 ? 2 : 3;                      // stages: more would leave fewer CTAs resident (11008 x 4096, 1 row: 3 11.7 us, 5 23.7;
                                                                            // 32 rows: 2 19.6 us, 3 38.3)
    static constexpr int kX = kTile * kCodeRow, kScales = kX + 8 * kBlocks * kXRow, kBytes = kScales + kTile * kScaleRow;
};

template <typename T, int kGroup, int kBlocks>
__global__ void __launch_bounds__(kThreads) matmul_mma_kernel(const W4Args a)
{
    using S = Stage<kGroup, kBlocks>;
    extern __shared__ __align__(16) uint8_t smem[];
    const uint32_t rank = cluster_ctarank(), split = gridDim.x;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, quad = lane & 3, row = lane >> 2;
    const int o0 = blockIdx.y * kTile, t0 = blockIdx.z * 8 * kBlocks;
    // whole chunks for every CTA, so that its scales begin at a boundary
    const int all = (a.groups + S::kGroups - 1) / S::kGroups, c0 = (int)(all * rank / split), c1 = (int)(all * (rank + 1) / split);
    const int chunks = c1 - c0, g0 = c0 * S::kGroups, g1 = min(c1 * S::kGroups, a.groups);
    cluster_arrive();
    pdl_wait();
    pdl_launch_dependents();
    // rows and outputs beyond the end are computed like the last ones and not written
    const T *scales = static_cast<const T *>(a.scales) + (long long)min(o0 + tid, a.outputs - 1) * a.groups + g0;
    // scales of an output's chunk are one copy where rows of scales allow it; otherwise as many loads as there are groups, each of which meets 32 lines
    const bool wide = a.groups % S::kGroups == 0 && reinterpret_cast<uintptr_t>(a.scales) % S::kScaleRow == 0;
    auto fetch = [&](int c, int at) {                                       // chunk c into stage `at`
        uint8_t *stage = smem + at * S::kBytes;
        const int i0 = (g0 + c * S::kGroups) * kGroup, n = min(kChunk, (g1 - g0 - c * S::kGroups) * kGroup);
#pragma unroll
        for (int i = tid; i < 8 * kBlocks * (kChunk / 8); i += kThreads) {
            const int r = i / (kChunk / 8), piece = i % (kChunk / 8);
            const bool there = piece * 8 < n;
            copy_async<16>(stage + S::kX + r * S::kXRow + piece * 16,
                           static_cast<const T *>(a.x) + (long long)min(t0 + r, a.rows - 1) * a.x_row + i0 + (there ? piece * 8 : 0), there);
        }
        if (wide) {
            copy_async<S::kScaleRow>(stage + S::kScales + tid * S::kScaleRow, scales + c * S::kGroups, true);
        } else {
#pragma unroll
            for (int g = 0; g < S::kGroups; ++g)
                if (c * S::kGroups + g < g1 - g0) reinterpret_cast<T *>(stage + S::kScales + tid * S::kScaleRow)[g] = __ldg(scales + c * S::kGroups + g);
        }
        // eight lanes a row, its 128 bytes
        const int piece = tid & 7;
        const bool there = piece * 32 < n;
#pragma unroll
        for (int i = 0; i < kTile / 16; ++i) {
            const int r = i * 16 + tid / 8;
            copy_async<16>(stage + r * S::kCodeRow + piece * 16, a.codes + ((long long)min(o0 + r, a.outputs - 1) * a.inputs + i0) / 2 + (there ? piece * 16 : 0), there);
        }
    };
    float sum[2][kBlocks][4];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[m][n][i] = 0.f;

    const int stages = a.stages;
    for (int c = 0; c < stages; ++c) {
        if (c < chunks) fetch(c, c);
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    int at = 0;
#pragma unroll 1
    for (int c = 0; c < chunks; ++c) {
        wait_copies(stages - 1);
        __syncthreads();
        const uint8_t *stage = smem + at * S::kBytes;
        const T *held = reinterpret_cast<const T *>(stage + S::kScales);    // [output][group]
        const int groups = min(S::kGroups, g1 - g0 - c * S::kGroups);
        const uint8_t *codes = stage + (warp * 32 + row) * S::kCodeRow + quad * (S::kWords * 4);
        const uint8_t *x = stage + S::kX + row * S::kXRow + quad * (S::kWords * 16);
#pragma unroll
        for (int g = 0; g < S::kGroups; ++g) {                              // unrolled: a group's chain is long, and they overlap
            if (g >= groups) break;
            float acc[2][kBlocks][4];
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int n = 0; n < kBlocks; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[m][n][i] = 0.f;
#pragma unroll
            for (int j = 0; j < kGroup / S::kSub; ++j) {
                const int at = g * kGroup + j * S::kSub;
                uint32_t w[4][S::kWords];
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    const uint8_t *p = codes + m * 8 * S::kCodeRow + at / 2;
                    if constexpr (S::kWords == 2) {
                        const uint2 v = *reinterpret_cast<const uint2 *>(p);
                        w[m][0] = v.x;
                        w[m][1] = v.y;
                    } else {
                        w[m][0] = *reinterpret_cast<const uint32_t *>(p);
                    }
                }
#pragma unroll
                for (int k = 0; k < S::kWords; ++k) {
                    uint32_t b[kBlocks][4];
#pragma unroll
                    for (int n = 0; n < kBlocks; ++n) {
                        // the pairs (0, 4), (1, 5), (2, 6), (3, 7) of eight inputs, as the codes come
                        const uint4 v = *reinterpret_cast<const uint4 *>(x + n * 8 * S::kXRow + at * 2 + k * 16);
                        b[n][0] = __byte_perm(v.x, v.z, 0x5410);
                        b[n][1] = __byte_perm(v.x, v.z, 0x7632);
                        b[n][2] = __byte_perm(v.y, v.w, 0x5410);
                        b[n][3] = __byte_perm(v.y, v.w, 0x7632);
                    }
                    uint32_t p[4][4];
#pragma unroll
                    for (int m = 0; m < 4; ++m) unpack<T>(w[m][k], p[m]);
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int n = 0; n < kBlocks; ++n) {
                            const uint32_t lo[4] = {p[2 * m][0], p[2 * m + 1][0], p[2 * m][1], p[2 * m + 1][1]};
                            const uint32_t hi[4] = {p[2 * m][2], p[2 * m + 1][2], p[2 * m][3], p[2 * m + 1][3]};
                            mma16816<T>(acc[m][n], lo, b[n][0], b[n][1]);
                            mma16816<T>(acc[m][n], hi, b[n][2], b[n][3]);
                        }
                }
            }
            float s[4];
#pragma unroll
            for (int m = 0; m < 4; ++m) s[m] = (float)held[(warp * 32 + m * 8 + row) * S::kGroups + g];
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int n = 0; n < kBlocks; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[m][n][i] = fmaf(s[2 * m + (i >> 1)], acc[m][n][i], sum[m][n][i]);
        }
        if (chunks > stages) {                                              // the stage is used again
            __syncthreads();
            if (c + stages < chunks) fetch(c + stages, at);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++at == stages) at = 0;
    }
    // An output's parts go to the CTA whose share of the tile it is, [rank][row][output of the share]: a barrier less than fetching them there.
    const int share = kTile / split;
    float *part = reinterpret_cast<float *>(smem + stages * S::kBytes);
    cluster_wait();                                                 // every CTA has begun
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        const int o = warp * 32 + m * 16;                           // the 16 outputs from here are of one share
        const uint32_t there = mapa_rank(smem_u32(part + rank * (8 * kBlocks) * share + o % share + row), o / share);
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there + 4 * ((n * 8 + quad * 2 + (i & 1)) * share + (i >> 1) * 8)), "f"(sum[m][n][i]) : "memory");
    }
    cluster_sync_all();
    const int rows = min(8 * kBlocks, a.rows - t0);
    for (int i = tid; i < rows * share; i += kThreads) {
        const int t = t0 + i / share, o = o0 + rank * share + i % share;
        float y = part[i];
#pragma unroll
        for (uint32_t c = 1; c < kMaxSplit; ++c) y = c < split ? y + part[c * (8 * kBlocks) * share + i] : y;
        if (o >= a.outputs) continue;
        if (a.relu && y < 0.f) y = 0.f;
        if (a.residual) y += (float)static_cast<const T *>(a.residual)[t * a.residual_row + o];
        static_cast<T *>(a.out)[t * a.out_row + o] = from_float<T>(y);
    }
}

// ---- quantisation --------------------------------------------------------------------------------------------------
// One thread a group of an output; neighbours take neighbouring outputs (or, of weights that lie by outputs, groups).  Done once for a matrix, and not
// made fast: 4096 x 11008 with adjacent outputs 99 us, with adjacent inputs 397 (90 MB in: 14 us).
template <typename T, int kGroup>
__global__ void __launch_bounds__(128)
quantise_kernel(const T *__restrict__ w, long long w_in, long long w_out, int groups, int outputs, uint8_t *__restrict__ codes,
                T *__restrict__ scales)
{
    const long long i = (long long)blockIdx.x * 128 + threadIdx.x;
    if (i >= (long long)groups * outputs) return;
    const bool by_output = w_out <= w_in;
    const long long o = by_output ? i % outputs : i / groups, g = by_output ? i / outputs : i % groups;
    const T *v = w + o * w_out + g * kGroup * w_in;
    float most = 0.f;
    for (int k = 0; k < kGroup; ++k) most = fmaxf(most, fabsf((float)v[k * w_in]));
    const T scale = from_float<T>(__fdiv_rn(most, 7.f));
    const float s = (float)scale;
    scales[o * groups + g] = scale;
    uint32_t *out = reinterpret_cast<uint32_t *>(codes + (o * groups + g) * (kGroup / 2));
    for (int k = 0; k < kGroup; k += 8) {
        uint32_t word = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float c = s > 0.f ? fminf(fmaxf(rintf(__fdiv_rn((float)v[(k + j) * w_in], s)), -8.f), 7.f) : 0.f;
            word |= (uint32_t)((int)c + 8) << (4 * j);
        }
        out[k / 8] = word;
    }
}

template <typename F> cudaError_t by_group(int group, F &&f)
{
    return group == 32 ? f(std::integral_constant<int, 32>{}) : group == 64 ? f(std::integral_constant<int, 64>{}) : f(std::integral_constant<int, 128>{});
}

template <typename T, int kGroup, int kBlocks> cudaError_t launch_mma(const W4Args &args, cudaStream_t stream)
{
    using S = Stage<kGroup, kBlocks>;
    const int tiles = (args.outputs + kTile - 1) / kTile, steps = (args.rows + 8 * kBlocks - 1) / (8 * kBlocks);
    // CTAs that share a tile's inputs: eight, with 256 inputs at least (4096 x 4096, 1 row: eight 6.1 us, four 7.0, one 16; 4096 x 32000: 29.7, 36, 34)
    int split = kMaxSplit;
    while (split > 1 && args.inputs / split < kChunk) split /= 2;
    W4Args a = args;
    const int chunks = ((a.groups + S::kGroups - 1) / S::kGroups + split - 1) / split;
    a.stages = chunks < S::kMost ? chunks : S::kMost;
    const size_t smem = a.stages * (size_t)S::kBytes + 8 * kBlocks * kTile * sizeof(float);
    static std::atomic<bool> ready[64];                             // by device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev >= 64 || !ready[dev])) {
        e = cudaFuncSetAttribute(matmul_mma_kernel<T, kGroup, kBlocks>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 S::kMost * S::kBytes + 8 * kBlocks * kTile * (int)sizeof(float));
        if (e == cudaSuccess && dev < 64) ready[dev] = true;
    }
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.gridDim = dim3(split, tiles, steps);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, matmul_mma_kernel<T, kGroup, kBlocks>, a);
}

template <typename T> cudaError_t launch_type(const W4Args &a, int group, cudaStream_t stream)
{
    return by_group(group, [&](auto g) {
        constexpr int kGroup = decltype(g)::value;
        return a.rows <= 8    ? launch_mma<T, kGroup, 1>(a, stream)
               : a.rows <= 16 ? launch_mma<T, kGroup, 2>(a, stream)
                              : launch_mma<T, kGroup, 4>(a, stream);
    });
}

}  // namespace

cudaError_t launch_w4_matmul(const W4Args &a, int dtype, int group, cudaStream_t stream)
{
    return dtype == kF16 ? launch_type<__half>(a, group, stream) : launch_type<__nv_bfloat16>(a, group, stream);
}

cudaError_t launch_w4_quantise(const void *w, long long w_in, long long w_out, int inputs, int outputs, int dtype, int group,
                               uint8_t *codes, void *scales, cudaStream_t stream)
{
    return by_group(group, [&](auto g) {
        constexpr int kGroup = decltype(g)::value;
        const int groups = inputs / kGroup;
        const unsigned grid = (unsigned)(((long long)groups * outputs + 127) / 128);
        if (dtype == kF16)
            quantise_kernel<__half, kGroup><<<grid, 128, 0, stream>>>(static_cast<const __half *>(w), w_in, w_out, groups, outputs, codes, static_cast<__half *>(scales));
        else
            quantise_kernel<__nv_bfloat16, kGroup><<<grid, 128, 0, stream>>>(static_cast<const __nv_bfloat16 *>(w), w_in, w_out, groups, outputs, codes,
                                                                           static_cast<__nv_bfloat16 *>(scales));
        return cudaGetLastError();
    });
}

}  // namespace dresd
