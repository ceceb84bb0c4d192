// out = beta out + alpha A B^T of two operands in 4-bit blocks (kimad_mx4.cuh) on the fifth-generation tensor cores.
//
// tcgen05.mma of kind mxf4 takes the codes as they lie in the operands (K-major, two to a byte), 64 values of the summed axis at a time, and
// the two scales a line that go with them; products of codes are exact, scaled by powers of two and added in binary32 in tensor memory.  The
// scales' tiles (128 lines by 4 blocks, 512 bytes) are in the order that tensor memory wants: lane r % 32, column r / 32, a byte per block.
//
// A CTA makes a tile of 128 by 128 outputs: one warp brings stages of 256 values (128 bytes) of 128 lines of either operand by TMA, 128-byte
// swizzled, and their scales by bulk copies; one thread of another warp copies the scales to tensor memory and issues the products; four warps
// take the sums out (32 lines each), turn slabs of 32 by 32 around in shared memory and update the output in lines of consecutive elements,
// whatever its alignment.  Two CTAs share an SM: one's outputs are written beside the other's products.
// Lines behind the operand's last and bytes behind a line's last block are filled with zeros by TMA: code 0 times any scale that is there
// is 0, and the scales that are not there are 0 too.
// Waits are bounded (kMxWaitClocks): a CTA whose wait ran out stores nothing, waits for its copies, frees its tensor memory and sets the status.
#pragma once
#include <cuda.h> // CUtensorMap

#include "kimad_mx4.cuh"

namespace kimad {

constexpr int kMxStages = 3;
constexpr uint32_t kMxStageK = 256;                  // values of the summed axis in a stage
constexpr uint32_t kMxOperandStage = 128 * 128;      // bytes of codes of an operand in a stage
constexpr uint32_t kMxScaleStage = 2 * 512;          // ... and of scales
constexpr uint32_t kMxStageBytes = 2 * kMxOperandStage + 2 * kMxScaleStage;
constexpr uint32_t kMxProductSmem = 1024 + kMxStages * kMxStageBytes;
constexpr int kMxProductThreads = 192;               // warps 0-3 outputs, 4 copies, 5 products
constexpr uint32_t kMxTmemCols = 256;                // 128 of sums, 16 of scales a stage
constexpr long long kMxWaitClocks = 1ll << 31;       // about a second

// Instruction descriptor of kind mxf4: E2M1 by E2M1, scales UE8M0, K-major, N = 128 (bits 17-22, in eights), M = 128 (bits 27-28, in 128s).
// The two scales of a product lie in bytes 0-1 or 2-3 of their column (bits 4-5 for B, 29-30 for A).
constexpr uint32_t kMxIdesc = (1u << 7) | (1u << 10) | ((128u / 8u) << 17) | (1u << 23) | (1u << 27);
__device__ __forceinline__ uint32_t mx_idesc(uint32_t half) { return kMxIdesc | (half * 2u) << 4 | (half * 2u) << 29; }

// Shared-memory descriptors: lines of 128 bytes, 128-byte swizzle, eight lines to 1024 bytes; and for the scales no swizzle, eight rows of 16 bytes to 128.
__device__ __forceinline__ uint64_t mx_desc_codes(uint32_t addr) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__device__ __forceinline__ uint64_t mx_desc_scales(uint32_t addr) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)(128 >> 4) << 16 | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.b32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
// Bounded: false when the phase has not ended within the limit or another warp of the CTA has given up.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile uint32_t* failed) {
    if (mbar_try(bar, parity)) return true;
    const long long began = clock64();
    while (!mbar_try(bar, parity))
        if (*failed || clock64() - began > kMxWaitClocks) { *failed = 1; return false; }
    return true;
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(x),
                 "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_copy_scales(uint32_t tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void tc_mma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
                 "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa),
                 "r"(sb), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tc_load32(uint32_t (&r)[32], uint32_t addr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
                   "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

struct MxProduct {
    float* out;
    uint64_t ld, batch_stride;
    const uint8_t *scales_a, *scales_b;
    MxOperand a, b;
    float alpha, beta;
    int32_t* status;
};

__global__ void __launch_bounds__(kMxProductThreads)
k_mx4_product(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ MxProduct p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t s_bar[2 * kMxStages + 1];
    __shared__ uint32_t s_tmem;
    __shared__ volatile uint32_t s_failed;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t bar = smem_u32(s_bar), smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    float* slabs = reinterpret_cast<float*>(smem_raw + (smem - smem_u32(smem_raw)));
    auto full = [&](uint32_t s) { return bar + 8 * s; };
    auto empty = [&](uint32_t s) { return bar + 8 * (kMxStages + s); };
    const uint32_t done = bar + 8 * (2 * kMxStages);
    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < kMxStages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        mbar_init(done, 1);
        s_failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(kMxTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s_tmem;
    pdl_wait();

    const uint32_t bt = blockIdx.x % p.b.line_tiles, at = blockIdx.x / p.b.line_tiles % p.a.line_tiles;
    const uint32_t n = blockIdx.x / p.b.line_tiles / p.a.line_tiles;
    const uint32_t rounds = (p.a.blocks + kMxStageK / kMxBlock - 1) / (kMxStageK / kMxBlock), tiles = p.a.block_tiles;
    uint32_t r = 0; // rounds whose copies, or whose products, have been issued
    if (warp == 4 && lane == 0) {
        const uint8_t* sa = p.scales_a + ((uint64_t)n * p.a.line_tiles + at) * tiles * 512;
        const uint8_t* sb = p.scales_b + ((uint64_t)n * p.b.line_tiles + bt) * tiles * 512;
        for (; r < rounds; ++r) {
            const uint32_t s = r % kMxStages, to = smem + s * kMxStageBytes;
            if (r >= kMxStages && !mbar_wait(empty(s), (r / kMxStages - 1) & 1u, &s_failed)) break;
            const uint32_t scale_bytes = min(tiles - 2 * r, 2u) * 512u;
            mbar_expect(full(s), 2 * kMxOperandStage + 2 * scale_bytes);
            tma_load_3d(to, &map_a, (int)(r * 128), (int)(at * kMxTile), (int)n, full(s));
            tma_load_3d(to + kMxOperandStage, &map_b, (int)(r * 128), (int)(bt * kMxTile), (int)n, full(s));
            bulk_load(to + 2 * kMxOperandStage, sa + (uint64_t)r * 1024, scale_bytes, full(s));
            bulk_load(to + 2 * kMxOperandStage + kMxScaleStage, sb + (uint64_t)r * 1024, scale_bytes, full(s));
        }
    } else if (warp == 5 && lane == 0) {
        for (; r < rounds; ++r) {
            const uint32_t s = r % kMxStages, from = smem + s * kMxStageBytes, scales = tmem + 128 + 16 * s;
            if (!mbar_wait(full(s), (r / kMxStages) & 1u, &s_failed)) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t products = min((p.a.blocks - r * 8 + 1) / 2, 4u); // of 64 values, two blocks, each
            for (uint32_t t = 0; 2 * t < products; ++t) {
                tc_copy_scales(scales + 4 * t, mx_desc_scales(from + 2 * kMxOperandStage + 512 * t));
                tc_copy_scales(scales + 8 + 4 * t, mx_desc_scales(from + 2 * kMxOperandStage + kMxScaleStage + 512 * t));
            }
            for (uint32_t k = 0; k < products; ++k)
                tc_mma_mxf4(tmem, mx_desc_codes(from + 32 * k), mx_desc_codes(from + kMxOperandStage + 32 * k), mx_idesc(k & 1u), scales + 4 * (k >> 1),
                            scales + 8 + 4 * (k >> 1), r + k > 0);
            tc_commit(empty(s));
        }
        tc_commit(done);
    }
    __syncwarp();
    if (warp < 4) {
        const bool fine = mbar_wait(done, 0, &s_failed) && !s_failed;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (fine) {
            float* slab = slabs + warp * 32 * 33;
            const uint32_t row0 = at * kMxTile + warp * 32, col0 = bt * kMxTile;
            float* out = p.out + n * p.batch_stride + (uint64_t)row0 * p.ld + col0;
            const uint32_t rows = row0 < p.a.lines ? min(p.a.lines - row0, 32u) : 0u;
            for (uint32_t c = 0; c < kMxTile && col0 + c < p.b.lines; c += 32) {
                uint32_t v[32];
                if (rounds) tc_load32(v, tmem + (warp * 32 << 16) + c);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 32; ++i) slab[lane * 33 + i] = rounds ? __uint_as_float(v[i]) : 0.f;
                __syncwarp();
                const bool in = col0 + c + lane < p.b.lines;
                float was[32];
#pragma unroll
                for (uint32_t i = 0; i < 32; ++i) was[i] = p.beta != 0.f && in && i < rows ? out[i * p.ld + c + lane] : 0.f;
#pragma unroll
                for (uint32_t i = 0; i < 32; ++i) {
                    float x = __fmul_rn(p.alpha, slab[i * 33 + lane]);
                    if (p.beta != 0.f) x = __fmaf_rn(p.beta, was[i], x);
                    if (in && i < rows) out[i * p.ld + c + lane] = x;
                }
            }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncthreads();
    if (s_failed) { // what was issued still writes to this CTA's shared and tensor memory
        if (threadIdx.x == 0 && p.status) *p.status = KIMAD_ERR_TIMEOUT;
        const long long began = clock64();
        if (warp == 4 && lane == 0)
            for (uint32_t i = r > kMxStages ? r - kMxStages : 0; i < r; ++i)
                while (!mbar_try(full(i % kMxStages), (i / kMxStages) & 1u) && clock64() - began < kMxWaitClocks) {}
        if (warp == 5 && lane == 0)
            while (!mbar_try(done, 0) && clock64() - began < kMxWaitClocks) {}
        __syncwarp();
    }
    if (warp == 5) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kMxTmemCols) : "memory");
    }
}

} // namespace kimad
