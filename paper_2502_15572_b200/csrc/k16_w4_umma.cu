// K16 -- products with 4-bit weights for many rows (a chunk of drafts, a piece of a prompt), on tcgen05.
//
// What K15 computes, with the same arithmetic: codes minus 8 and activations are multiplied as they are, exact in the activations' type, and the
// scale meets a group's sum in fp32.  A CTA has 256 outputs (two halves of 128, the M of the instruction) and up to 128 rows (its N):
//
//     A   codes minus 8 in TMEM, written by the warps that unpack them: a thread owns an output; four slots of 64 inputs, two a half
//     B   activations in shared memory as TMA lays them (128-byte swizzle, K-major), used by both halves
//     D   three blocks of 128 columns in turn; a block is the sum of ONE group, which other warps take out, scale and add to the
//         sums in their registers (an output a thread, up to 128 rows) while the tensor core works on the next two
//
// Weights rounded to 16 bits with their scales would need no second step, but add an error as large as the result's own rounding; that step's
// instructions (an fma for every sum of a group, sixteen columns at a time) fit beside the unpacking as long as groups are not small.
//
// Bound: 101 rows of 11008 x 4096 27.5 us (floor 5.5): 16 tiles, each by a cluster of 6 (16 of more do not fit at once), so that a CTA goes through its 15 blocks
// of inputs one after the other, each of some 2000 cycles (unpack, store to TMEM, products, take out), and then joins.  2047 rows of 4096 x 11008 175 us (1.05 PFLOP/s,
// 0.63 of the measured rate; 204 as one call among others, when the power limit lowers the clock): some 1900 cycles a block, of which products take 1024;
// the unit for logic and shifts is busy for half of the time, and the rest are handovers between the roles.
//
// Roles: warp 0 loads (lane 0: codes and activations of 128 inputs a stage), warps 1 and 2 issue the products of a half each, warps 4-11 unpack,
// warps 12-19 scale and add.
// With few tiles the CTAs of a cluster split the inputs and add their parts up in the order of their ranks; with many, CTAs are persistent.
#include <atomic>
#include <type_traits>

#include "kv_plan.cuh"

namespace dresd {
namespace {

constexpr int kThreads = 640, kOutputs = 256, kTileRows = 128, kBlock = 128;     // inputs of a stage
constexpr int kCodeBytes = kOutputs * kBlock / 2;
constexpr int kMaxStages = 8, kMaxSplit = 8;
constexpr int kSmemBytes = 232448;
constexpr uint32_t kColumnsA = 384;                            // of the first slot; D at 0, 128, 256
constexpr int kControl = 40, kUnpack = 56, kAdd = 160;         // registers of the roles' warps
static_assert(kControl + 2 * kUnpack + 2 * kAdd <= 5 * 96, "what a CTA is launched with: 5 warpgroups of 96 a thread");

__device__ unsigned int g_expired;                             // waits that ran out; see w4_expired()

struct UmmaArgs {
    W4Args w;
    int n;                      // rows of a tile, a multiple of 16
    int row_tiles, tiles;
    int blocks;                 // of 128 inputs
    int split, stages;
    long long wait_cycles;
    int lose_stage;             // test hook: the first CTA never receives its stage (value - 1)
};

struct Shared {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t a_full[2][2], a_empty[2][2], drained;            // of a half's slots of 64 inputs
    // Of a half's own sums in turn, so that a warp that waits has seen the one three before; sum v of half h lies in block (2 v + h) % 3.
    uint64_t d_full[2][3], d_empty[2][3];
    uint32_t tmem;
};

__device__ __forceinline__ void umma_f16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Sixteen columns, waited for (in one piece: apart, every register is moved once more).
__device__ __forceinline__ void tmem_load16(uint32_t taddr, uint32_t *r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
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
// A warpgroup's registers per thread.
template <bool kMore, int kCount> __device__ __forceinline__ void set_registers()
{
    if constexpr (kMore) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kCount));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kCount));
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
// The eight codes of a word, minus 8, as pairs of T: nibbles become bits of the mantissas of powers of two, the lower one of a byte the lowest bits
// (fp16 2048 + 2 c, bf16 256 + 2 c), the upper one those above them (fp16 128 + 2 c; bf16, which has fewer, moved down by one: 32 + 2 c).  Half of
// that minus 1032, 136, 72, 24 is exact, and an fma: additions of halves go to the unit that permutes bytes, and that is the busiest one here.
template <typename T> __device__ __forceinline__ void unpack(uint32_t w, uint32_t *p);
template <> __device__ __forceinline__ void unpack<__half>(uint32_t w, uint32_t *p)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t two = (__byte_perm(w, w, 0x1111 * k) & 0x00F0000Fu) | 0x58006800u, half = 0x38003800u, less = 0xD480E408u;
        const __half2 r = __hfma2(*reinterpret_cast<const __half2 *>(&two), *reinterpret_cast<const __half2 *>(&half), *reinterpret_cast<const __half2 *>(&less));
        p[k] = *reinterpret_cast<const uint32_t *>(&r);
    }
}
template <> __device__ __forceinline__ void unpack<__nv_bfloat16>(uint32_t w, uint32_t *p)
{
    const uint32_t down = w >> 1;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t two = (__byte_perm(w, down, 0x4400 + 0x1111 * k) & 0x0078000Fu) | 0x42004380u, half = 0x3F003F00u, less = 0xC1C0C308u;
        const __nv_bfloat162 r = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&two), *reinterpret_cast<const __nv_bfloat162 *>(&half),
                                         *reinterpret_cast<const __nv_bfloat162 *>(&less));
        p[k] = *reinterpret_cast<const uint32_t *>(&r);
    }
}

template <typename T> __device__ __forceinline__ void unpack(const uint4 &w, uint32_t *p)
{
    unpack<T>(w.x, p);
    unpack<T>(w.y, p + 4);
    unpack<T>(w.z, p + 8);
    unpack<T>(w.w, p + 12);
}

template <typename T, int kGroup>
__global__ void __launch_bounds__(kThreads, 1)
matmul_umma_kernel(const __grid_constant__ CUtensorMap code_map, const __grid_constant__ CUtensorMap x_map, const __grid_constant__ UmmaArgs a)
{
    constexpr int kGroups = kBlock / kGroup;                    // of a block
    extern __shared__ uint8_t smem_raw[];
    __shared__ Shared sh;
    const int slab = a.n * 128, stage_bytes = kCodeBytes + 2 * slab;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long wl = a.wait_cycles;
    const int rank = a.split > 1 ? (int)cluster_ctarank() : 0;
    const int tile0 = blockIdx.x / a.split, tile_step = gridDim.x / a.split;
    const int b0 = (int)((long long)a.blocks * rank / a.split), b1 = (int)((long long)a.blocks * (rank + 1) / a.split);
    const int groups = min(b1 * kGroups, a.w.groups) - b0 * kGroups;       // of this CTA
    uint8_t *stages = smem_raw + (-smem_u32(smem_raw) & 1023u);

    if (warp == 0) {
        if (lane < a.stages) {
            mbar_init(&sh.full[lane], 1);
            mbar_init(&sh.empty[lane], 8 + 2);                  // the unpacking warps, the halves' products
        }
        if (lane < 2) {
            mbar_init(&sh.a_full[0][lane], 4);
            mbar_init(&sh.a_full[1][lane], 4);
            mbar_init(&sh.a_empty[0][lane], 1);
            mbar_init(&sh.a_empty[1][lane], 1);
        }
        if (lane < 3) {
            mbar_init(&sh.d_full[0][lane], 1);
            mbar_init(&sh.d_full[1][lane], 1);
            mbar_init(&sh.d_empty[0][lane], 4);
            mbar_init(&sh.d_empty[1][lane], 4);
        }
        if (lane == 3) mbar_init(&sh.drained, 2);
        mbar_fence_init();
        if (lane == 4) {
            tma_prefetch_desc(&code_map);
            tma_prefetch_desc(&x_map);
        }
    } else if (warp == 3) {
        tmem_alloc(&sh.tmem, 512);
        tmem_relinquish();
    }
    pdl_wait();
    pdl_launch_dependents();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;

    if (warp < 4) {
        set_registers<false, kControl>();
        if (warp == 0 && lane == 0) {
            int it = 0;
            bool ok = true;
#pragma unroll 1
            for (int tile = tile0; tile < a.tiles && ok; tile += tile_step) {
                const int o = tile / a.row_tiles * kOutputs, t = tile % a.row_tiles * a.n;
#pragma unroll 1
                for (int b = b0; b < b1; ++b, ++it) {
                    const int s = it % a.stages;
                    if (it >= a.stages && !mbar_wait(&sh.empty[s], (it / a.stages - 1) & 1, wl)) {
                        ok = false;
                        break;
                    }
                    uint8_t *dst = stages + s * stage_bytes;
                    mbar_arrive_expect_tx(&sh.full[s], (uint32_t)stage_bytes);
                    if (a.lose_stage > 0 && blockIdx.x == 0 && it == a.lose_stage - 1) continue;
                    tma_load_2d(dst, &code_map, b * (kBlock / 2), o, &sh.full[s]);
                    tma_load_2d(dst + kCodeBytes, &x_map, b * kBlock, t, &sh.full[s]);
                    tma_load_2d(dst + kCodeBytes + slab, &x_map, b * kBlock + 64, t, &sh.full[s]);
                }
            }
            // what is on its way arrives before the CTA ends
            for (int i = max(0, it - a.stages); i < it; ++i)
                if (!mbar_wait(&sh.full[i % a.stages], (i / a.stages) & 1, wl)) ok = false;
            if (!ok) atomicAdd(&g_expired, 1u);
        } else if (warp == 1 || warp == 2) {
            // One thread issues, the warp goes along: code that only one thread reaches takes 90 cycles an instruction, a product of 128 rows 64.  A
            // warp to each half: the waits and commits of a block take one warp 2000 cycles, its products 1024.
            constexpr uint32_t kFmt = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
            const uint32_t idesc = (1u << 4) | (kFmt << 7) | (kFmt << 10) | ((uint32_t)(a.n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
            const bool issuer = elect_one();
            const uint32_t slab_step = slab >> 4;
            const int half = warp - 1;
            const uint32_t a_at = tmem + kColumnsA + half * 64;
            int v = 0, d = half, s = 0, s_phase = 0, a_phase = 0;        // the half's sums, block of the next one, stage
            bool ok = true;
            auto wait = [&](uint64_t *bar, uint32_t phase) { return __all_sync(0xFFFFFFFFu, mbar_wait(bar, phase, wl)); };
#pragma unroll 1
            for (int tile = tile0; tile < a.tiles && ok; tile += tile_step)
#pragma unroll 1
                for (int b = b0; b < b1; ++b) {
                    const int here = min(kGroups, groups - (b - b0) * kGroups);
                    const uint64_t x_desc = make_desc(smem_u32(stages + s * stage_bytes + kCodeBytes));
                    if (!(ok = wait(&sh.full[s], s_phase))) break;
                    uint32_t d_at = 0;
#pragma unroll
                    for (int k = 0; k < kBlock / 16; ++k) {
                        const bool there = k / (kGroup / 16) < here;
                        if (k % (kGroup / 16) == 0 && there) {
                            d_at = tmem + (uint32_t)d * kTileRows;
                            // the sum three before in all: of the other half
                            const int e = v - 2 + half;
                            if (e >= 0 && ok) ok = wait(&sh.d_empty[half ^ 1][e % 3], (e / 3) & 1);
                        }
                        if (k % 4 == 0 && ok) ok = wait(&sh.a_full[half][k / 4], a_phase);
                        if (k % 4 == 0 || k % (kGroup / 16) == 0) tc_fence_after();
                        if (issuer && ok && there)
                            umma_f16_ta(d_at, a_at + k * 8, x_desc + (k / 4 * slab_step + 2 * (k & 3)), idesc, k % (kGroup / 16) != 0);
                        if (k % 4 == 3 && issuer && ok) tc_commit(&sh.a_empty[half][k / 4]);
                        if ((k + 1) % (kGroup / 16) == 0 && there) {
                            if (issuer && ok) tc_commit(&sh.d_full[half][v % 3]);
                            ++v;
                            d = d == 0 ? 2 : d - 1;             // (2 v + half) % 3
                        }
                    }
                    a_phase ^= 1;
                    if (!ok) break;
                    if (issuer) tc_commit(&sh.empty[s]);
                    if (++s == a.stages) {
                        s = 0;
                        s_phase ^= 1;
                    }
                }
            // no product may be running when TMEM is given back
            if (issuer) tc_commit(&sh.drained);
            if (!wait(&sh.drained, 0)) ok = false;
            if (!ok && lane == 0) atomicAdd(&g_expired, 1u);
        }
    } else if (warp < 12) {
        set_registers<false, kUnpack>();
        const int half = (warp - 4) >> 2, quarter = warp & 3, r = half * 128 + quarter * 32 + lane;
        const uint32_t to = tmem + kColumnsA + half * 64 + ((uint32_t)(quarter * 32) << 16);
        // 64 bytes of a row, which TMA has swizzled by 64 bytes
        const uint8_t *row = stages + r * 64;
        const int swizzle = ((r >> 1) & 3) * 16;
        int s = 0, s_phase = 0, a_phase = 1;                    // (the phase before the first one counts as complete)
        bool ok = true;
#pragma unroll 1
        for (int tile = tile0; tile < a.tiles && ok; tile += tile_step)
#pragma unroll 1
            for (int b = b0; b < b1; ++b) {
                if (!__all_sync(0xFFFFFFFFu, mbar_wait(&sh.full[s], s_phase, wl))) { ok = false; break; }
                uint4 w[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) w[c] = *reinterpret_cast<const uint4 *>(row + s * stage_bytes + (16 * c ^ swizzle));
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.empty[s]);
                if (++s == a.stages) {
                    s = 0;
                    s_phase ^= 1;
                }
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    uint32_t p[16];
                    unpack<T>(w[2 * q], p);                     // before the slot is free
                    if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&sh.a_empty[half][q], a_phase, wl));
                    tc_fence_after();
                    if (ok) tmem_st16(to + 32 * q, p);
                    unpack<T>(w[2 * q + 1], p);
                    if (ok) tmem_st16(to + 32 * q + 16, p);
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (ok && lane == 0) mbar_arrive(&sh.a_full[half][q]);
                }
                a_phase ^= 1;
                if (!ok) break;
            }
        if (!ok && lane == 0) atomicAdd(&g_expired, 1u);
    } else {
        set_registers<true, kAdd>();
        const int half = (warp - 12) >> 2, quarter = warp & 3, r = half * 128 + quarter * 32 + lane;
        const uint32_t from = tmem + ((uint32_t)(quarter * 32) << 16);
        int i_full = 0, full_phase = 0, d = half;               // this half's sums: of three barriers in turn, block
        bool ok = true;
#pragma unroll 1
        for (int tile = tile0; tile < a.tiles && ok; tile += tile_step) {
            const int o = tile / a.row_tiles * kOutputs + r, t0 = tile % a.row_tiles * a.n;
            const T *scales = static_cast<const T *>(a.w.scales) + (long long)min(o, a.w.outputs - 1) * a.w.groups + b0 * kGroups;
            float sum[kTileRows];
#pragma unroll
            for (int i = 0; i < kTileRows; ++i) sum[i] = 0.f;
            T next = __ldg(scales);
#pragma unroll 1
            for (int g = 0; g < groups; ++g) {
                const float scale = (float)next;
                if (g + 1 < groups) next = __ldg(scales + g + 1);
                if (!__all_sync(0xFFFFFFFFu, mbar_wait(&sh.d_full[half][i_full], full_phase, wl))) { ok = false; break; }
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < kTileRows / 16; ++c) {
                    if (c * 16 >= a.n) break;
                    uint32_t x[16];
                    tmem_load16(from + d * kTileRows + 16 * c, x);
#pragma unroll
                    for (int i = 0; i < 16; ++i) sum[16 * c + i] = fmaf(scale, __uint_as_float(x[i]), sum[16 * c + i]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.d_empty[half][i_full]);
                d = d == 0 ? 2 : d - 1;
                if (++i_full == 3) {
                    i_full = 0;
                    full_phase ^= 1;
                }
            }
            if (!ok) break;
            if (a.split > 1) {
                // [row][output], where the stages were: when all products are done, the other half's too
                if (!__all_sync(0xFFFFFFFFu, mbar_wait(&sh.drained, 0, wl))) { ok = false; break; }
                float *part = reinterpret_cast<float *>(stages);
#pragma unroll
                for (int c = 0; c < kTileRows / 16; ++c) {
                    if (c * 16 >= a.n) break;
#pragma unroll
                    for (int i = 16 * c; i < 16 * c + 16; ++i) part[i * kOutputs + r] = sum[i];
                }
            } else if (o < a.w.outputs) {
                T *out = static_cast<T *>(a.w.out) + t0 * a.w.out_row + o;
                const T *residual = a.w.residual ? static_cast<const T *>(a.w.residual) + t0 * a.w.residual_row + o : nullptr;
                const int rows = min(a.n, a.w.rows - t0);
                if (a.w.relu) {
#pragma unroll
                    for (int i = 0; i < kTileRows; ++i) sum[i] = sum[i] < 0.f ? 0.f : sum[i];
                }
                // (checks and products of a row's address, all in one loop: a tenth of a long call)
#pragma unroll
                for (int c = 0; c < kTileRows / 16; ++c) {
                    if (c * 16 >= rows) break;
                    if (residual) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            if (c * 16 + i < rows) sum[16 * c + i] += (float)*residual;
                            residual += a.w.residual_row;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        if (c * 16 + i < rows) *out = (T)sum[16 * c + i];
                        out += a.w.out_row;
                    }
                }
            }
        }
        if (!ok && lane == 0) atomicAdd(&g_expired, 1u);
    }
    __syncwarp();
    if (a.split > 1) {
        // one tile a cluster: its parts, each CTA a share of the rows, by the warps with registers for it
        cluster_sync_all();
        const int o0 = tile0 / a.row_tiles * kOutputs, t0 = tile0 % a.row_tiles * a.n;
        const float *part = reinterpret_cast<const float *>(stages);
#pragma unroll 1
        for (int i = warp < 12 ? a.n * (kOutputs / 4) : rank * 256 + tid - 384; i < a.n * (kOutputs / 4); i += a.split * 256) {
            const int t = t0 + i / (kOutputs / 4), o = o0 + i % (kOutputs / 4) * 4;
            if (t >= a.w.rows || o >= a.w.outputs) continue;
            float4 v[kMaxSplit];
#pragma unroll
            for (int c = 0; c < kMaxSplit; ++c)
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                             : "=f"(v[c].x), "=f"(v[c].y), "=f"(v[c].z), "=f"(v[c].w)
                             : "r"(mapa_rank(smem_u32(part + 4 * i), min(c, a.split - 1))) : "memory");
            float y[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
            for (int c = 1; c < kMaxSplit; ++c) {
                if (c >= a.split) break;
                y[0] += v[c].x;
                y[1] += v[c].y;
                y[2] += v[c].z;
                y[3] += v[c].w;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (o + j >= a.w.outputs) break;
                if (a.w.relu && y[j] < 0.f) y[j] = 0.f;
                if (a.w.residual) y[j] += (float)static_cast<const T *>(a.w.residual)[t * a.w.residual_row + o + j];
                static_cast<T *>(a.w.out)[t * a.w.out_row + o + j] = (T)y[j];
            }
        }
        cluster_sync_all();                                     // the others may still read this CTA's part
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 3) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// CTAs (clusters of `split`) that are resident at once.
template <typename T, int kGroup> cudaError_t resident(int split, int smem, int sms, int *clusters)
{
    static std::atomic<int> known[64][kMaxSplit + 1];           // by device; + 1
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    *clusters = dev < 64 ? known[dev][split].load() - 1 : -1;
    if (*clusters >= 0) return cudaSuccess;
    e = cudaFuncSetAttribute(matmul_umma_kernel<T, kGroup>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    if (split == 1) {
        *clusters = sms;
    } else {
        cudaLaunchConfig_t cfg{};
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = split;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.gridDim = dim3(split);
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = smem;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(clusters, matmul_umma_kernel<T, kGroup>, &cfg);
        if (e != cudaSuccess) return e;
    }
    if (dev < 64) known[dev][split].store(*clusters + 1);
    return cudaSuccess;
}

template <typename T, int kGroup>
cudaError_t launch(const CUtensorMap &code_map, const CUtensorMap &x_map, UmmaArgs a, int sms, cudaStream_t stream)
{
    constexpr int kRing = kSmemBytes - 1024 - (int)sizeof(Shared) - 64;
    const int stage = kCodeBytes + a.n * 256, smem = kRing + 1024;
    a.stages = min(kRing / stage, kMaxStages);
    // Inputs are split over a cluster when tiles are few: the split with the least work in a row, where a join counts as four blocks.
    long long best = -1;
    int clusters = 0;
    for (int split = 1; split <= min(kMaxSplit, a.blocks); ++split) {
        int room = 0;
        const cudaError_t e = resident<T, kGroup>(split, smem, sms, &room);
        if (e != cudaSuccess) return e;
        if (room < 1) continue;
        const long long rounds = (a.tiles + room - 1) / room, cost = rounds * ((a.blocks + split - 1) / split + (split > 1 ? 4 : 0));
        if (best < 0 || cost < best) {
            best = cost;
            a.split = split;
            clusters = room;
        }
        if (a.tiles >= sms) break;
    }
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = a.split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.gridDim = dim3(a.split > 1 ? a.tiles * a.split : min(a.tiles, clusters));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = a.split > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, matmul_umma_kernel<T, kGroup>, code_map, x_map, a);
}

template <typename T>
cudaError_t by_group(int group, const CUtensorMap &code_map, const CUtensorMap &x_map, const UmmaArgs &a, int sms, cudaStream_t stream)
{
    return group == 32   ? launch<T, 32>(code_map, x_map, a, sms, stream)
           : group == 64 ? launch<T, 64>(code_map, x_map, a, sms, stream)
                         : launch<T, 128>(code_map, x_map, a, sms, stream);
}

}  // namespace

int w4_umma_rows(int rows)
{
    const int tiles = (rows + kTileRows - 1) / kTileRows;
    return ((rows + tiles - 1) / tiles + 15) / 16 * 16;
}

cudaError_t launch_w4_umma(const CUtensorMap &code_map, const CUtensorMap &x_map, const W4Args &w, int dtype, int group, long long wait_cycles,
                           int lose_stage, int sms, cudaStream_t stream)
{
    UmmaArgs a{};
    a.w = w;
    a.n = w4_umma_rows(w.rows);
    a.row_tiles = (w.rows + a.n - 1) / a.n;
    a.tiles = (w.outputs + kOutputs - 1) / kOutputs * a.row_tiles;
    a.blocks = (w.inputs + kBlock - 1) / kBlock;
    a.wait_cycles = wait_cycles;
    a.lose_stage = lose_stage;
    return dtype == kF16 ? by_group<__half>(group, code_map, x_map, a, sms, stream) : by_group<__nv_bfloat16>(group, code_map, x_map, a, sms, stream);
}

cudaError_t w4_expired(unsigned int *count, cudaStream_t stream)
{
    *count = 0;
    const cudaError_t e = cudaMemcpyFromSymbolAsync(count, g_expired, sizeof *count, 0, cudaMemcpyDeviceToHost, stream);
    return e == cudaSuccess ? cudaStreamSynchronize(stream) : e;
}

}  // namespace dresd
