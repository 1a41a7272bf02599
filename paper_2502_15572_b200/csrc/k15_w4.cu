// K15 -- products with 4-bit weights and one scale for a group of inputs:
//     y[t][o] = sum_g s[o][g] sum_{i in g} (c[o][i] - 8) x[t][i]
// The inner sums multiply whole numbers -8 .. 7 and the activations, both exact in the activations' type, and are kept in fp32; the scale meets
// them there.  So a weight is never rounded, and a result is rounded once.
//
// A warp computes 32 outputs for up to 8 kBlocks rows with mma.sync, weights as the 16-row operand.  The order of inputs within an
// instruction is free, as long as both operands agree: a lane takes G / 4 consecutive codes of a row, as they lie in
// memory (4 lanes a row, 8 rows a load), and the same inputs of its row of activations.  No shared memory is involved until the
// end, when the CTAs of a cluster, which split the inputs, add their parts up in the order of their ranks.
#include <type_traits>

#include "kv_plan.cuh"

namespace dresd {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps, kTile = 32 * kWarps;      // outputs of a CTA
constexpr int kMaxSplit = 8;

// Codes of nibbles j and j + 4 of `w` (already moved to j = 0), minus 8, as a pair of T: the nibble in the low bits of the mantissa of 1024
// (fp16) or 128 (bf16) is that number plus the code.
template <typename T> __device__ __forceinline__ uint32_t code_pair(uint32_t w);
template <> __device__ __forceinline__ uint32_t code_pair<__half>(uint32_t w)
{
    const uint32_t u = (w & 0x000F000Fu) | 0x64006400u, c = 0x64086408u;      // 1024 + 8
    const __half2 r = __hsub2(*reinterpret_cast<const __half2 *>(&u), *reinterpret_cast<const __half2 *>(&c));
    return *reinterpret_cast<const uint32_t *>(&r);
}
template <> __device__ __forceinline__ uint32_t code_pair<__nv_bfloat16>(uint32_t w)
{
    const uint32_t u = (w & 0x000F000Fu) | 0x43004300u, c = 0x43084308u;      // 128 + 8
    const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&u), *reinterpret_cast<const __nv_bfloat162 *>(&c));
    return *reinterpret_cast<const uint32_t *>(&r);
}
template <typename T> __device__ __forceinline__ float scale_of(const void *scales, long long i)
{
    const T v = __ldg(static_cast<const T *>(scales) + i);
    if constexpr (std::is_same<T, __half>::value) return __half2float(v);
    else return __bfloat162float(v);
}
template <typename T> __device__ __forceinline__ T from_float(float x)
{
    if constexpr (std::is_same<T, __half>::value) return __float2half_rn(x);
    else return __float2bfloat16_rn(x);
}
template <typename T> __device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Eight codes a word: words of a lane's share of a group of one row, as one load.
template <int kWords> struct Words;
template <> struct Words<4> { typedef uint4 type; };
template <> struct Words<2> { typedef uint2 type; };
template <> struct Words<1> { typedef uint32_t type; };

template <typename T, int kGroup, int kBlocks>
__global__ void __launch_bounds__(kThreads) matmul_mma_kernel(const W4Args a)
{
    constexpr int kWords = kGroup / 32, kAhead = 512 / kGroup;      // groups whose codes are loaded together
    typedef typename Words<kWords>::type Load;
    extern __shared__ float part[];                                 // [8 kBlocks rows][kTile outputs]
    const uint32_t rank = cluster_ctarank(), split = gridDim.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane & 3, row = lane >> 2;
    const int o0 = blockIdx.y * kTile + warp * 32, t0 = blockIdx.z * 8 * kBlocks;
    const int g0 = (int)((long long)a.groups * rank / split), g1 = (int)((long long)a.groups * (rank + 1) / split);
    pdl_wait();
    pdl_launch_dependents();
    // rows and outputs beyond the end are computed like the last ones and not written
    const uint8_t *codes[4];
    long long scale_row[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const long long o = min(o0 + m * 8 + row, a.outputs - 1);
        codes[m] = a.codes + o * (a.inputs / 2) + quad * (kGroup / 8);
        scale_row[m] = o * a.groups;
    }
    const T *x[kBlocks];
#pragma unroll
    for (int n = 0; n < kBlocks; ++n) x[n] = static_cast<const T *>(a.x) + (long long)min(t0 + n * 8 + row, a.rows - 1) * a.x_row + quad * (kGroup / 4);
    float sum[2][kBlocks][4];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[m][n][i] = 0.f;

    for (int g = g0; g < g1; g += kAhead) {
        Load w[kAhead][4];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
#pragma unroll
            for (int m = 0; m < 4; ++m)
                if (g + j < g1) w[j][m] = __ldg(reinterpret_cast<const Load *>(codes[m] + (long long)(g + j) * (kGroup / 2)));
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (g + j >= g1) break;
            float s[4], acc[2][kBlocks][4];
#pragma unroll
            for (int m = 0; m < 4; ++m) s[m] = scale_of<T>(a.scales, scale_row[m] + g + j);
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int n = 0; n < kBlocks; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[m][n][i] = 0.f;
#pragma unroll
            for (int k = 0; k < kWords; ++k) {
                uint32_t b[kBlocks][4];
#pragma unroll
                for (int n = 0; n < kBlocks; ++n) {
                    // the pairs (0, 4), (1, 5), (2, 6), (3, 7) of eight inputs, as the codes come
                    const uint4 v = __ldg(reinterpret_cast<const uint4 *>(x[n] + (long long)(g + j) * kGroup + k * 8));
                    b[n][0] = __byte_perm(v.x, v.z, 0x5410);
                    b[n][1] = __byte_perm(v.x, v.z, 0x7632);
                    b[n][2] = __byte_perm(v.y, v.w, 0x5410);
                    b[n][3] = __byte_perm(v.y, v.w, 0x7632);
                }
                uint32_t c[4][4];
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    const uint32_t word = reinterpret_cast<const uint32_t *>(&w[j][m])[k];
#pragma unroll
                    for (int p = 0; p < 4; ++p) c[m][p] = code_pair<T>(word >> (4 * p));
                }
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int n = 0; n < kBlocks; ++n) {
                        const uint32_t lo[4] = {c[2 * m][0], c[2 * m + 1][0], c[2 * m][1], c[2 * m + 1][1]};
                        const uint32_t hi[4] = {c[2 * m][2], c[2 * m + 1][2], c[2 * m][3], c[2 * m + 1][3]};
                        mma16816<T>(acc[m][n], lo, b[n][0], b[n][1]);
                        mma16816<T>(acc[m][n], hi, b[n][2], b[n][3]);
                    }
            }
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int n = 0; n < kBlocks; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[m][n][i] = fmaf(s[2 * m + (i >> 1)], acc[m][n][i], sum[m][n][i]);
        }
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                part[(n * 8 + quad * 2 + (i & 1)) * kTile + warp * 32 + m * 16 + (i >> 1) * 8 + row] = sum[m][n][i];
    cluster_sync_all();
    // results are shared out over the cluster; neighbours in a warp are neighbours in memory
    for (int i = rank * kThreads + threadIdx.x; i < 8 * kBlocks * kTile; i += split * kThreads) {
        const int t = t0 + i / kTile, o = blockIdx.y * kTile + i % kTile;
        if (t >= a.rows || o >= a.outputs) continue;
        float y = 0.f;
        for (uint32_t c = 0; c < split; ++c) {
            float v;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(mapa_rank(smem_u32(part + i), c)) : "memory");
            y += v;
        }
        if (a.relu && y < 0.f) y = 0.f;
        if (a.residual) y += (float)static_cast<const T *>(a.residual)[t * a.residual_row + o];
        static_cast<T *>(a.out)[t * a.out_row + o] = from_float<T>(y);
    }
    cluster_sync_all();                                             // the others may still read this CTA's part
}

// ---- quantisation --------------------------------------------------------------------------------------------------
// One thread a group of an output; neighbours take neighbouring outputs (or, of weights that lie by outputs, groups).
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

template <typename T, int kGroup, int kBlocks> cudaError_t launch_mma(const W4Args &a, int sms, cudaStream_t stream)
{
    const int tiles = (a.outputs + kTile - 1) / kTile, steps = (a.rows + 8 * kBlocks - 1) / (8 * kBlocks);
    // CTAs that share a tile's inputs: until there are four a SM, each with 512 inputs at least
    int split = 1;
    while (split < kMaxSplit && (long long)tiles * steps * split < 4LL * sms && a.inputs / (split * 2) >= 512) split *= 2;
    const size_t smem = sizeof(float) * 8 * kBlocks * kTile;
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

template <typename T> cudaError_t launch_type(const W4Args &a, int group, int sms, cudaStream_t stream)
{
    return by_group(group, [&](auto g) {
        constexpr int kGroup = decltype(g)::value;
        return a.rows <= 8    ? launch_mma<T, kGroup, 1>(a, sms, stream)
               : a.rows <= 16 ? launch_mma<T, kGroup, 2>(a, sms, stream)
                              : launch_mma<T, kGroup, 4>(a, sms, stream);
    });
}

}  // namespace

cudaError_t launch_w4_matmul(const W4Args &a, int dtype, int group, int sms, cudaStream_t stream)
{
    return dtype == kF16 ? launch_type<__half>(a, group, sms, stream) : launch_type<__nv_bfloat16>(a, group, sms, stream);
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
