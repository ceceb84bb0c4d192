// out = beta out + alpha A B^T of two operands in 4-bit blocks (kimad_mx4.cuh) on the fifth-generation tensor cores.
//
// tcgen05.mma of kind mxf4 takes the codes as they lie in the operands (K-major, two to a byte), 64 values of the summed axis at a time, and
// the two scales a line that go with them; products of codes are exact, scaled by powers of two and added in binary32 in tensor memory.  The
// scales' tiles (128 lines by 4 blocks, 512 bytes) are in the order that tensor memory wants: lane r % 32 (in all four quarters of it), column
// r / 32, a byte per block.
//
// One warp brings stages of 256 values (128 bytes) of the operands' lines by TMA, 128-byte swizzled; four warps bring the scales to tensor memory, a
// quarter each (copies by tcgen05.cp wait in line with the products: a stage of 128 by 128 then took 590 clocks of an SM, 256 of them products); one
// lane of another warp issues the products; further warps take the sums out and update the output.
// k_mx4_product_pairs has two SMs for a tile, k_mx4_product_parts several for parts of the summed axis of one.
// Lines behind the operand's last and bytes behind a line's last block are filled with zeros by TMA: code 0 times any scale that is there
// is 0, and the scales that are not there are 0 too.
// Waits are bounded (kMxWaitClocks, and kMxRoundClocks a round where a whole sum is waited for): a CTA whose wait ran out stores nothing more, waits for
// its copies, frees its tensor memory and sets the device's status, and the caller's if there is one.
#pragma once
#include <cuda.h> // CUtensorMap

#include "kimad_mx4.cuh"

namespace kimad {

constexpr uint32_t kMxStageK = 256;                  // values of the summed axis in a stage
constexpr uint32_t kMxOperandStage = 128 * 128;      // bytes of codes of an operand in a stage
constexpr long long kMxWaitClocks = 1ll << 31;       // about a second: the limit of a wait, by default, and of those after a failure
constexpr long long kMxRoundClocks = 8192;           // what a wait for a whole sum is given besides, a round of kMxStageK values: they take about 500

// Instruction descriptor of kind mxf4: E2M1 by E2M1, scales UE8M0, K-major, N (bits 17-22, in eights), M (bits 27-28, in 128s).
// The two scales of a product lie in bytes 0-1 or 2-3 of their column (bits 4-5 for B, 29-30 for A).
KIMAD_HD constexpr uint32_t mx_idesc(uint32_t m, uint32_t n, uint32_t half) {
    return (1u << 7) | (1u << 10) | ((n / 8u) << 17) | (1u << 23) | ((m / 128u) << 27) | (half * 2u) << 4 | (half * 2u) << 29;
}

// Shared-memory descriptor: lines of 128 bytes, 128-byte swizzle, eight lines to 1024 bytes.
__device__ __forceinline__ uint64_t mx_desc_codes(uint32_t addr) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
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
// ... for a phase that another CTA of the cluster arrives in.
__device__ __forceinline__ bool mbar_try_cluster(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.b32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
// Waits of whole warps, bounded: false, for all lanes, when the phase has not ended within the limit or another warp of the CTA has given up.
struct MxWait {
    volatile uint32_t* flag;
    long long clocks;
    __device__ __forceinline__ bool failed() const { return __any_sync(0xffffffffu, *flag != 0); }
};
template <bool CLUSTER = false> __device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, const MxWait& w) {
    auto look = [&] { return CLUSTER ? mbar_try_cluster(bar, parity) : mbar_try(bar, parity); };
    bool ended = look();
    if (__all_sync(0xffffffffu, ended)) return true;
    const long long began = clock64();
    while (!ended && !(ended = look()))
        if (*w.flag || clock64() - began > w.clocks) { *w.flag = 1; break; }
    return __all_sync(0xffffffffu, ended);
}
__device__ __forceinline__ void tma_prefetch(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(x),
                 "r"(y), "r"(z), "r"(bar) : "memory");
}
// A load into this CTA's shared memory that is counted on a barrier of either CTA of its pair.
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(x),
                 "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void tc_store16(uint32_t addr, const uint4 (&v)[4]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr), "r"(v[0].x), "r"(v[0].y),
                 "r"(v[0].z), "r"(v[0].w), "r"(v[1].x), "r"(v[1].y), "r"(v[1].z), "r"(v[1].w), "r"(v[2].x), "r"(v[2].y), "r"(v[2].z), "r"(v[2].w), "r"(v[3].x),
                 "r"(v[3].y), "r"(v[3].z), "r"(v[3].w) : "memory");
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, int x, int y, int z, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(src) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// All but the `most` latest stores of this thread have read their memory.
template <int most> __device__ __forceinline__ void tma_stores_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(most) : "memory"); }
__device__ __forceinline__ void tma_stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// GROUP: CTAs whose tensor cores take one product together.
template <int GROUP> __device__ __forceinline__ void tc_mma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
    if (GROUP == 1)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
                     "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa),
                     "r"(sb), "r"(accumulate) : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
                     "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa),
                     "r"(sb), "r"(accumulate) : "memory");
}
// Arrival when all products issued so far are done: on this CTA's barrier, or on both CTAs' of a pair.
template <int GROUP> __device__ __forceinline__ void tc_commit(uint32_t bar) {
    if (GROUP == 1) asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((unsigned short)3) : "memory");
}
__device__ __forceinline__ void tc_load32(uint32_t (&r)[32], uint32_t addr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
                   "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// One lane of a warp, the same one every time.  (With a lane's number in its place, and roles by a thread's number, the compiler does not see that addresses
// and descriptors are the same for the whole warp, and every copy and product takes about 100 clocks to issue.)
__device__ __forceinline__ bool one_lane() {
    uint32_t one;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.b32 %0, 1, 0, p;\n}" : "=r"(one));
    return one != 0;
}
__device__ __forceinline__ uint32_t warp_number() { return __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0); }

// A place in a ring of barriers and the parity of its present phase.
template <uint32_t N> struct MxRing {
    uint32_t s = 0, parity = 0;
    __device__ __forceinline__ void next() {
        if (++s == N) { s = 0; parity ^= 1u; }
    }
};

__device__ int32_t g_mx4_status; // KIMAD_ERR_TIMEOUT once a wait of any product has run out on the device (kimad_mx4_product_status)
__device__ __forceinline__ void mx_report(int32_t* status) {
    g_mx4_status = KIMAD_ERR_TIMEOUT;
    if (status) *status = KIMAD_ERR_TIMEOUT;
}

struct MxProduct {
    float* out;
    uint64_t ld, batch_stride;
    const uint8_t *scales_a, *scales_b;
    MxOperand a, b;
    float alpha, beta;
    int32_t* status;
    long long wait_clocks;
    uint32_t withhold; // codes are not copied, so that waits run out
};

// A warp's part of the output, 32 rows by slabs of 32 columns.  A lane has a row of the sums, as tensor memory gives them.  Where the output's rows lie on
// 32 bytes and a slab is whole, a lane updates its row by four accesses of 32 bytes (whole sectors), whose old values can be fetched ahead; elsewhere the slab
// is turned around in shared memory (`buf`, 32 x 33) and updated in lines of consecutive elements, any alignment and any edge.
struct MxOutput {
    float* at;   // row 0, column 0
    float* mine; // this lane's row
    uint64_t ld;
    uint32_t rows, cols; // that are there
    float alpha, beta;
    uint32_t lane;
    bool aligned;
    __device__ __forceinline__ MxOutput(const MxProduct& p, uint32_t n, uint32_t row, uint32_t col, uint32_t most_cols, uint32_t lane_)
        : at(p.out + n * p.batch_stride + (uint64_t)row * p.ld + col), ld(p.ld), alpha(p.alpha), beta(p.beta), lane(lane_) {
        mine = at + lane * ld;
        rows = row < p.a.lines ? min(p.a.lines - row, 32u) : 0u;
        cols = col < p.b.lines ? min(p.b.lines - col, most_cols) : 0u;
        if (!KIMAD_CHECK(rows == 0 || cols == 0 || ((uint64_t)row + rows <= p.a.lines && (uint64_t)col + cols <= p.b.lines && p.b.lines <= ld), 10)) rows = cols = 0;
        aligned = reinterpret_cast<uintptr_t>(at) % 32 == 0 && ld % 8 == 0;
    }
    __device__ __forceinline__ bool whole(uint32_t slab) const { return aligned && 32 * slab + 32 <= cols; }
    // A slab's old values: a lane's row where it is whole, otherwise a lane's column.
    __device__ __forceinline__ void fetch(uint32_t slab, float (&was)[32]) const {
        if (beta == 0.f) return;
        if (whole(slab)) {
            if (lane < rows) {
#pragma unroll
                for (uint32_t i = 0; i < 32; i += 8) mx_load8(mine + 32 * slab + i, *reinterpret_cast<float(*)[8]>(&was[i]));
            }
        } else {
            const float* from = at + 32 * slab + lane;
            const uint32_t here = 32 * slab + lane < cols ? rows : 0u;
#pragma unroll
            for (uint32_t i = 0; i < 32; ++i, from += ld) was[i] = i < here ? __ldcs(from) : 0.f;
        }
    }
    __device__ __forceinline__ float update(uint32_t sum, float was) const {
        const float x = __fmul_rn(alpha, __uint_as_float(sum));
        return beta != 0.f ? __fmaf_rn(beta, was, x) : x;
    }
    __device__ __forceinline__ void put(uint32_t slab, const uint32_t (&sums)[32], const float (&was)[32], float* buf) const {
        if (whole(slab)) {
            if (lane < rows) {
#pragma unroll
                for (uint32_t i = 0; i < 32; i += 8) {
                    float x[8];
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j) x[j] = update(sums[i + j], was[i + j]);
                    mx_store8(mine + 32 * slab + i, x);
                }
            }
            return;
        }
        if (32 * slab >= cols || rows == 0) return;
        __syncwarp();
#pragma unroll
        for (uint32_t i = 0; i < 32; ++i) buf[lane * 33 + i] = __uint_as_float(sums[i]);
        __syncwarp();
        float x[32]; // all of them before the first store: the compiler cannot tell that the output is not in shared memory
#pragma unroll
        for (uint32_t i = 0; i < 32; ++i) x[i] = buf[i * 33 + lane];
        float* to = at + 32 * slab + lane;
        const uint32_t here = 32 * slab + lane < cols ? rows : 0u;
#pragma unroll
        for (uint32_t i = 0; i < 32; ++i, to += ld)
            if (i < here) asm volatile("st.global.f32 [%0], %1;" ::"l"(to), "f"(update(__float_as_uint(x[i]), was[i])) : "memory");
    }
};

// The scales of two blocks of four for this lane's quarter: a line of each 32, 16 bytes.  0 where there are none.
__device__ __forceinline__ uint4 mx_scale_words(const uint8_t* tile, uint32_t chunk, uint32_t chunks, uint32_t lane) {
    return chunk < chunks ? __ldg(reinterpret_cast<const uint4*>(tile + (uint64_t)chunk * 512) + lane) : make_uint4(0, 0, 0, 0);
}

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint4 shared4(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
__device__ __forceinline__ uint2 shared2(uint32_t at) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
    return v;
}
// ... and of another CTA of the cluster.
__device__ __forceinline__ uint32_t shared_of(uint32_t at, uint32_t rank) {
    uint32_t there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(rank));
    return there;
}
// A copy from here to there, counted on the barrier there.
__device__ __forceinline__ void far_copy(uint32_t there, uint32_t src, uint32_t bytes, uint32_t bar_there) {
    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(there), "r"(src), "r"(bytes), "r"(bar_there) : "memory");
}
__device__ __forceinline__ uint32_t mx_add(uint32_t a, uint32_t b) { return __float_as_uint(__fadd_rn(__uint_as_float(a), __uint_as_float(b))); }

// ---- Parts.  Where there are few tiles and a long sum, a cluster of two or four CTAs shares a tile of 128 by 128 (gridDim.z of them): each takes a part of the
// summed axis, copies its sums of a part of the tile's columns to each of the others' shared memory, and adds up those of its own part, in the order of the
// CTAs.  (Also where nothing is summed at all.)  256 x 2048 outputs over 8192 values: 9.7 us with two
// CTAs a tile, 12.9 by pairs of SMs.  With the sums read from the others' memory instead of copied there by the copy engine it took 13.5, with plain stores
// to it 11.4.
constexpr int kMxPartStages = 5;
constexpr uint32_t kMxPartStageBytes = 2 * kMxOperandStage;
constexpr uint32_t kMxJoin = 4 * 4 * 4096; // bytes of a tile's sums
constexpr uint32_t kMxPartSmem = 1024 + kMxPartStages * kMxPartStageBytes + kMxJoin;
constexpr int kMxPartThreads = 192;    // warps 0-3 scales and outputs, 4 copies, 5 products
constexpr uint32_t kMxPartCols = 256;  // of tensor memory: 128 of sums, 16 of scales a stage
static_assert(kMxPartSmem <= 227 * 1024 && 128 + 16 * kMxPartStages <= kMxPartCols, "memory");

// A slab's sums over all parts, in their order: this CTA's own are in `sums`, the others' in shared memory.
template <uint32_t PARTS> __device__ __forceinline__ void mx_join(uint32_t slab, uint32_t part, uint32_t lane, uint32_t (&sums)[32]) {
#pragma unroll
    for (uint32_t c = 0; c < 8; ++c) {
        uint4 v[PARTS];
#pragma unroll
        for (uint32_t z = 0; z < PARTS; ++z)
            v[z] = z == part ? make_uint4(sums[4 * c], sums[4 * c + 1], sums[4 * c + 2], sums[4 * c + 3]) : shared4(slab + 4096 * z * (4 / PARTS) + ((c ^ (lane & 7u)) << 4));
#pragma unroll
        for (uint32_t z = 1; z < PARTS; ++z)
            v[0] = make_uint4(mx_add(v[0].x, v[z].x), mx_add(v[0].y, v[z].y), mx_add(v[0].z, v[z].z), mx_add(v[0].w, v[z].w));
        sums[4 * c] = v[0].x;
        sums[4 * c + 1] = v[0].y;
        sums[4 * c + 2] = v[0].z;
        sums[4 * c + 3] = v[0].w;
    }
}

__global__ void __launch_bounds__(kMxPartThreads, 1)
k_mx4_product_parts(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ MxProduct p) {
    extern __shared__ uint8_t smem_raw[];
    constexpr uint32_t S = kMxPartStages;
    __shared__ __align__(8) uint64_t s_bar[3 * S + 2];
    __shared__ uint32_t s_tmem;
    __shared__ volatile uint32_t s_failed;
    const MxWait wait{&s_failed, p.wait_clocks};
    const uint32_t warp = warp_number(), lane = threadIdx.x & 31;
    const uint32_t bar = smem_u32(s_bar), smem = (smem_u32(smem_raw) + 1023u) & ~1023u, parts = gridDim.z, part = blockIdx.z;
    const uint32_t full = bar, empty = bar + 8 * S, scaled = bar + 16 * S, done = bar + 24 * S, joined = done + 8; // a stage's copies, products, scales; all products; all parts' sums
    const uint32_t bt = blockIdx.x % p.b.line_tiles, at = blockIdx.x / p.b.line_tiles % p.a.line_tiles;
    const uint32_t n = blockIdx.x / p.b.line_tiles / p.a.line_tiles;
    const uint32_t all_rounds = (p.a.blocks + kMxStageK / kMxBlock - 1) / (kMxStageK / kMxBlock), tiles = p.a.block_tiles;
    const uint32_t most = (all_rounds + parts - 1) / parts, first = min(part * most, all_rounds), rounds = min(all_rounds - first, most); // of this CTA
    uint32_t r = 0; // rounds whose copies, or whose products, have been issued
    MxRing<S> q;
    auto bring = [&] { // the next stage's codes
        const uint32_t to = smem + q.s * kMxPartStageBytes, ready = full + 8 * q.s;
        if (one_lane()) {
            mbar_expect(ready, kMxPartStageBytes);
            tma_load_3d(to, &map_a, (int)((first + r) * 128), (int)(at * kMxTile), (int)n, ready);
            tma_load_3d(to + kMxOperandStage, &map_b, (int)((first + r) * 128), (int)(bt * kMxTile), (int)n, ready);
        }
        ++r;
        q.next();
    };
    if (warp == 4) { // the first copies are under way before the rest of the CTA is ready
        if (rounds && one_lane()) { tma_prefetch(&map_a); tma_prefetch(&map_b); }
        if (lane < 3 * S + 2) mbar_init(bar + 8 * lane, lane >= 2 * S && lane < 3 * S ? 4u : 1u); // (in the order of their places)
        s_failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        __syncwarp();
        if (parts > 1 && one_lane()) mbar_expect(joined, kMxJoin / parts * (parts - 1));
        pdl_wait();
        while (r < min(rounds, 2u) && !p.withhold) bring();
    }
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(kMxPartCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); // (waited for before anything is sent to another CTA)
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s_tmem;
    pdl_wait();

    float was[2][32];
    const MxOutput o(p, n, at * kMxTile + warp * 32, bt * kMxTile, kMxTile, lane); // (of warps 0-3)
    const uint32_t mine = tmem + (warp * 32 << 16);
    bool fine = false;
    if (warp == 4) {
        while (r < rounds && !p.withhold) {
            if (r >= S && !mbar_wait(empty + 8 * q.s, q.parity ^ 1u, wait)) break;
            bring();
        }
    } else if (warp == 5) {
        for (; r < rounds; ++r, q.next()) {
            const uint32_t scales = tmem + kMxTile + 16 * q.s;
            const uint64_t a = mx_desc_codes(smem + q.s * kMxPartStageBytes), b = mx_desc_codes(smem + q.s * kMxPartStageBytes + kMxOperandStage);
            if (!mbar_wait(scaled + 8 * q.s, q.parity, wait)) break; // ... which the warps that stored them have waited for `full` with
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t products = min((p.a.blocks - (first + r) * 8 + 1) / 2, 4u); // of 64 values, two blocks, each
            if (one_lane()) {
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k)
                    if (k < products) tc_mma_mxf4<1>(tmem, a + 2 * k, b + 2 * k, mx_idesc(128, 128, k & 1u), scales + 4 * (k >> 1), scales + 8 + 4 * (k >> 1), r + k > 0);
                tc_commit<1>(empty + 8 * q.s);
            }
        }
        if (one_lane()) tc_commit<1>(done);
    } else {
        const uint8_t* sa = p.scales_a + ((uint64_t)n * p.a.line_tiles + at) * tiles * 512;
        const uint8_t* sb = p.scales_b + ((uint64_t)n * p.b.line_tiles + bt) * tiles * 512;
        auto load = [&](uint32_t i, uint4 (&v)[4]) {
#pragma unroll
            for (uint32_t k = 0; k < 2; ++k) {
                v[k] = mx_scale_words(sa, 2 * (first + i) + k, tiles, lane);
                v[2 + k] = mx_scale_words(sb, 2 * (first + i) + k, tiles, lane);
            }
        };
        auto store = [&](const uint4 (&v)[4]) {
            if (!mbar_wait(full + 8 * q.s, q.parity, wait)) return false; // (and so the products that used the scales' place before are done)
            __syncwarp();
            tc_store16(mine + kMxTile + 16 * q.s, v);
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (one_lane()) mbar_arrive(scaled + 8 * q.s);
            q.next();
            return true;
        };
        uint4 v0[4], v1[4]; // two rounds under way
        load(0, v0);
        load(1, v1);
        o.fetch(part, was[0]); // behind the scales, which the products wait for
        if (part + parts < 4) o.fetch(part + parts, was[1]);
        for (uint32_t i = 0; i < rounds; i += 2) {
            if (!store(v0)) break;
            load(i + 2, v0);
            if (i + 1 >= rounds || !store(v1)) break;
            load(i + 3, v1);
        }
        fine = mbar_wait(done, 0, wait) && !wait.failed();
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    }
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    // Sums that the CTAs exchange: slabs of 32 by 32, a warp's four behind each other (CTA 0's for this one, CTA 1's, ..), sixteen bytes c of row i at c ^ (i % 8).
    // They leave from where the stages were; a CTA's own stay in tensor memory.
    const uint32_t in = smem + S * kMxPartStageBytes + warp * 4 * 4096, out = smem + warp * 4 * 4096;
    float* buf = reinterpret_cast<float*>(smem_raw + (smem - smem_u32(smem_raw)) + kMxJoin) + warp * 32 * 33;
    if (warp < 4 && fine && parts > 1) {
#pragma unroll 1
        for (uint32_t slab = 0; slab < 4; ++slab) {
            if (slab % parts == part) continue;
            uint32_t sums[32];
            if (rounds) tc_load32(sums, mine + 32 * slab);
#pragma unroll
            for (uint32_t c = 0; c < 8; ++c)
                asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(out + 4096 * slab + lane * 128 + ((c ^ (lane & 7u)) << 4)), "r"(rounds ? sums[4 * c] : 0u),
                             "r"(rounds ? sums[4 * c + 1] : 0u), "r"(rounds ? sums[4 * c + 2] : 0u), "r"(rounds ? sums[4 * c + 3] : 0u) : "memory");
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (one_lane()) {
            for (uint32_t slab = 0; slab < 4; ++slab)
                if (slab % parts != part)
                    far_copy(shared_of(in + 4096 * (part * (4 / parts) + slab / parts), slab % parts), out + 4096 * slab, 4096, shared_of(joined, slab % parts));
        }
        fine = mbar_wait(joined, 0, MxWait{&s_failed, p.wait_clocks + (long long)most * kMxRoundClocks}); // (the other CTAs may have started later)
        __syncwarp();
    }
    if (warp < 4 && fine) {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint32_t slab = part + i * parts;
            if (slab >= 4) break;
            uint32_t sums[32];
            if (rounds) tc_load32(sums, mine + 32 * slab);
            else {
#pragma unroll
                for (int k = 0; k < 32; ++k) sums[k] = 0;
            }
            if (parts == 4) mx_join<4>(in + 4096 * i + lane * 128, part, lane, sums);
            else if (parts == 2) mx_join<2>(in + 4096 * i + lane * 128, part, lane, sums);
            o.put(slab, sums, was[i & 1], buf);
            if (i < 2 && slab + 2 * parts < 4) o.fetch(slab + 2 * parts, was[i & 1]);
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (s_failed) { // what was issued still writes to this CTA's shared and tensor memory
        if (threadIdx.x == 0) mx_report(p.status);
        const long long began = clock64();
        if (warp == 4 && lane == 0)
            for (uint32_t i = r > S ? r - S : 0; i < r; ++i)
                while (!mbar_try(full + 8 * (i % S), (i / S) & 1u) && clock64() - began < kMxWaitClocks) {}
        if (warp == 5 && lane == 0)
            while (!mbar_try(done, 0) && clock64() - began < kMxWaitClocks) {}
        if (warp == 0 && lane == 0 && parts > 1)
            while (!mbar_try(joined, 0) && clock64() - began < kMxWaitClocks) {}
        __syncwarp();
    }
    cluster_sync(); // the copies from this CTA's memory have arrived
    if (warp == 5) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kMxPartCols) : "memory");
    }
}

// ---- Pairs.  Two CTAs (SMs) take tiles of 256 by kMxPairN together (cta_group::2): each holds 128 of A's lines and half of
// B's in shared memory, and both tensor cores read both halves.  An SM then reads 28 KB of codes per 256 values of a tile of 128 by 192 sums, where 128 by
// 128 alone needs 32: an SM takes 64 bytes per clock from L2, so a tile alone runs at half the products' rate at most.
// One CTA per SM stays for all its tiles; the sums are held twice, so that one tile's outputs are written beside the next one's products.  Outputs
// on 16 bytes (place, row distance and row length) come and go by TMA, slab by slab: the stores of eight warps are more than an SM gets rid of at once (about 16 bytes per clock when all
// write), and what waits in line behind them are the other warps' barriers, scales and products (stages took 2000 clocks beside them, 480 otherwise).
// Warps: 0-7 outputs (a quarter of the lines and half of the columns each), 8-11 scales to tensor memory, 12 copies of codes, 14 of scales (a copy takes
// almost 100 clocks to issue; all five of a stage in one warp are more than its products take), 13 products (in the pair's first CTA).
constexpr uint32_t kMxPairN = 192;
constexpr uint32_t kMxPairBytesB = kMxPairN / 2 * 128;
constexpr uint32_t kMxPairScales = 2 * 512; // bytes of a stage's scales of a tile of lines; of A's one and of B's two
constexpr uint32_t kMxPairStageBytes = kMxOperandStage + kMxPairBytesB + 3 * kMxPairScales;
KIMAD_HD constexpr uint32_t mx_pair_smem(uint32_t stages, uint32_t slabs) { return 1024 + stages * kMxPairStageBytes + 8 * slabs * 4096; }
constexpr int kMxPairThreads = 480;
constexpr uint32_t kMxPairScaleCols = 24; // of a stage: A's 2 x 4, B's 2 x 8 (6 in use)
static_assert(kMxPairStageBytes % 1024 == 0 && kMxPairN == 192, "shared memory; tc_store_scales");

// Arrival on the barrier of the pair's first CTA, for accesses to tensor memory and nothing else: they have been waited for (tcgen05.wait), and
// tcgen05.fence before the arrival and behind the other side's wait orders them, so that the arrival itself may be relaxed.  (With release it waits for every
// store under way, about 1000 clocks.)  The codes, which the copy engine writes to either CTA's shared memory, are counted on the first CTA's barrier
// themselves.
__device__ __forceinline__ void mbar_arrive_first(uint32_t bar) {
    asm volatile("{\n.reg .b32 a;\nmapa.shared::cluster.u32 a, %0, 0;\nmbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [a];\n}" ::"r"(bar) : "memory");
}
// A's eight words, and B's twelve at columns 8-13 and 16-21.
__device__ __forceinline__ void tc_store_scales(uint32_t addr, const uint4 (&a)[2], const uint2 (&b)[6]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(addr), "r"(a[0].x), "r"(a[0].y), "r"(a[0].z), "r"(a[0].w), "r"(a[1].x),
                 "r"(a[1].y), "r"(a[1].z), "r"(a[1].w) : "memory");
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%13,%13,%7,%8,%9,%10,%11,%12,%13,%13};" ::"r"(addr + 8), "r"(b[0].x), "r"(b[0].y),
                 "r"(b[1].x), "r"(b[1].y), "r"(b[2].x), "r"(b[2].y), "r"(b[3].x), "r"(b[3].y), "r"(b[4].x), "r"(b[4].y), "r"(b[5].x), "r"(b[5].y), "r"(0) : "memory");
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

struct MxPairTile {
    uint32_t row, col; // first output
    uint32_t n;        // matrix
    __device__ __forceinline__ MxPairTile(const MxProduct& p, uint32_t tile) {
        const uint32_t across = (p.b.lines + kMxPairN - 1) / kMxPairN, down = (p.a.lines + 255) / 256;
        col = tile % across * kMxPairN;
        row = tile / across % down * 256;
        n = tile / across / down;
    }
};

// S stages and, for each output warp, SLABS slabs under way.  More stages hide more of the copies' way from L2 (5632 x 5632 outputs over 8192 values with three,
// four, five stages: 131, 115, 108 us), more slabs more of the old values' (2 x 5632 x 2048 outputs and as many old values over 64 with two, three: 38.0, 34.4;
// over 1024: 41.2, 38.2).
template <uint32_t S, uint32_t SLABS>
__global__ void __launch_bounds__(kMxPairThreads, 1) __cluster_dims__(2, 1, 1)
k_mx4_product_pairs(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_out,
                    const __grid_constant__ MxProduct p, uint32_t all_tiles, uint32_t by_tma) {
    extern __shared__ uint8_t smem_raw[];
    static_assert(2 * kMxPairN + S * kMxPairScaleCols <= 512 && mx_pair_smem(S, SLABS) <= 227 * 1024 && SLABS <= kMxPairN / 64, "tensor memory, shared memory");
    __shared__ __align__(8) uint64_t s_bar[4 * S + 5 + 8 * SLABS];
    __shared__ uint32_t s_tmem;
    __shared__ volatile uint32_t s_failed;
    const MxWait wait{&s_failed, p.wait_clocks};
    const uint32_t warp = warp_number(), lane = threadIdx.x & 31, rank = cluster_rank();
    const uint32_t bar = smem_u32(s_bar), smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    // a stage's scales are here; its codes are, in both CTAs (first CTA); its scales are in tensor memory, in both CTAs (first CTA); its products are done; a
    // tile's products are done; its sums have been read, in both CTAs (first CTA); everything issued is done
    const uint32_t full = bar, codes = bar + 8 * S, ready = bar + 16 * S, empty = bar + 24 * S, done = bar + 32 * S, drained = done + 16, quit = done + 32,
                   old = quit + 8; // (an output warp's slabs of old values, SLABS each)
    if (warp == 12 && one_lane()) {
        tma_prefetch(&map_a);
        tma_prefetch(&map_b);
        if (by_tma) tma_prefetch(&map_out);
    }
    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < S; ++s) { mbar_init(full + 8 * s, 1); mbar_init(codes + 8 * s, 1); mbar_init(ready + 8 * s, 8); mbar_init(empty + 8 * s, 1); }
        for (uint32_t b = 0; b < 2; ++b) { mbar_init(done + 8 * b, 1); mbar_init(drained + 8 * b, 16); }
        mbar_init(quit, 1);
        for (uint32_t i = 0; i < 8 * SLABS; ++i) mbar_init(old + 8 * i, 1);
        s_failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 13) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s_tmem;
    pdl_wait();

    const uint32_t pair = blockIdx.x / 2, pairs = gridDim.x / 2;
    const uint32_t rounds = (p.a.blocks + kMxStageK / kMxBlock - 1) / (kMxStageK / kMxBlock), tiles = p.a.block_tiles;
    const MxWait whole{&s_failed, p.wait_clocks + (long long)rounds * kMxRoundClocks};
    uint32_t it = 0; // stages whose copies, or whose products, have been issued
    MxRing<S> q;
    if (warp == 12) {
        const uint32_t counted = shared_of(codes, 0);
        for (uint32_t tile = pair; tile < all_tiles && !p.withhold && !wait.failed(); tile += pairs) {
            const MxPairTile t(p, tile);
            for (uint32_t r = 0; r < rounds; ++r, ++it, q.next()) {
                const uint32_t to = smem + q.s * kMxPairStageBytes, there = counted + 8 * q.s;
                if (it >= S && !mbar_wait(empty + 8 * q.s, q.parity ^ 1u, wait)) break;
                if (one_lane()) { // (the second CTA's bytes may arrive before they are expected: the phase does not end before the first CTA's arrival)
                    if (rank == 0) mbar_expect(codes + 8 * q.s, 2 * (kMxOperandStage + kMxPairBytesB));
                    tma_load_3d_pair(to, &map_a, (int)(r * 128), (int)(t.row + rank * kMxTile), (int)t.n, there);
                    tma_load_3d_pair(to + kMxOperandStage, &map_b, (int)(r * 128), (int)(t.col + rank * (kMxPairN / 2)), (int)t.n, there);
                }
            }
        }
    } else if (warp == 14) {
        for (uint32_t tile = pair; tile < all_tiles && !wait.failed(); tile += pairs) {
            const MxPairTile t(p, tile);
            const uint32_t la = t.row / kMxTile + rank, lb = t.col / kMxTile; // tiles of lines whose scales are read
            const bool have_a = la < p.a.line_tiles, have_b = lb + 1 < p.b.line_tiles;
            const uint8_t* sa = p.scales_a + ((uint64_t)t.n * p.a.line_tiles + la) * tiles * 512;
            const uint8_t* sb = p.scales_b + ((uint64_t)t.n * p.b.line_tiles + lb) * tiles * 512;
            for (uint32_t r = 0; r < rounds; ++r, ++it, q.next()) {
                const uint32_t to = smem + q.s * kMxPairStageBytes + kMxOperandStage + kMxPairBytesB, here = full + 8 * q.s;
                if (!KIMAD_CHECK(2 * r < tiles && lb + have_b < p.b.line_tiles && la < p.a.line_tiles + !have_a, 10)) { s_failed = 1; break; }
                if (it >= S && !mbar_wait(empty + 8 * q.s, q.parity ^ 1u, wait)) break;
                if (one_lane()) {
                    const uint32_t bytes = min(tiles - 2 * r, 2u) * 512u;
                    mbar_expect(here, bytes * (1u + have_a + have_b));
                    if (have_a) bulk_load(to, sa + (uint64_t)r * 1024, bytes, here);
                    bulk_load(to + kMxPairScales, sb + (uint64_t)r * 1024, bytes, here);
                    if (have_b) bulk_load(to + 2 * kMxPairScales, sb + (uint64_t)tiles * 512 + (uint64_t)r * 1024, bytes, here);
                }
            }
        }
    } else if (warp == 13 && rank == 0) {
        MxRing<2> u; // places of sums
        uint32_t j = 0; // tiles of this pair
        for (uint32_t tile = pair; tile < all_tiles && !wait.failed(); tile += pairs, ++j, u.next()) {
            const uint32_t sums = tmem + u.s * kMxPairN;
            if (j >= 2 && !mbar_wait<true>(drained + 8 * u.s, u.parity ^ 1u, wait)) break;
            for (uint32_t r = 0; r < rounds; ++r, ++it, q.next()) {
                const uint32_t scales = tmem + 2 * kMxPairN + kMxPairScaleCols * q.s;
                const uint64_t a = mx_desc_codes(smem + q.s * kMxPairStageBytes), b = mx_desc_codes(smem + q.s * kMxPairStageBytes + kMxOperandStage);
                const uint32_t products = min((p.a.blocks - r * 8 + 1) / 2, 4u); // of 64 values, two blocks, each
                if (!mbar_wait(codes + 8 * q.s, q.parity, wait) || !mbar_wait<true>(ready + 8 * q.s, q.parity, wait)) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (one_lane()) {
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k)
                        if (k < products)
                            tc_mma_mxf4<2>(sums, a + 2 * k, b + 2 * k, mx_idesc(256, kMxPairN, k & 1u), scales + 4 * (k >> 1), scales + 8 + 8 * (k >> 1), r + k > 0);
                    tc_commit<2>(empty + 8 * q.s);
                }
            }
            if (wait.failed()) break; // (an unfinished tile is not announced: the other CTA may not know of the failure)
            if (one_lane()) tc_commit<2>(done + 8 * u.s);
        }
        if (wait.failed() && one_lane()) tc_commit<2>(quit);
    } else if (warp >= 8 && warp < 12) {
        const uint32_t mine = tmem + ((warp - 8) * 32 << 16) + 2 * kMxPairN;
        for (uint32_t tile = pair; tile < all_tiles && !wait.failed(); tile += pairs) {
            const MxPairTile t(p, tile);
            // this lane's words of B's lines, 64 by 64: the first ones may be a tile's second half
            const uint32_t b0 = kMxPairScales + t.col % kMxTile / 64 * 8, b1 = b0 & 8u ? 2 * kMxPairScales : b0 + 8, b2 = b0 & 8u ? b1 + 8 : 2 * kMxPairScales;
            for (uint32_t r = 0; r < rounds; ++r, q.next()) {
                const uint32_t from = smem + q.s * kMxPairStageBytes + kMxOperandStage + kMxPairBytesB + lane * 16;
                if (!mbar_wait(full + 8 * q.s, q.parity, wait)) break; // (and so the products that used the scales' place before are done)
                uint4 a[2];
                uint2 b[6];
#pragma unroll
                for (uint32_t k = 0; k < 2; ++k) {
                    a[k] = shared4(from + 512 * k);
                    b[3 * k] = shared2(from + 512 * k + b0);
                    b[3 * k + 1] = shared2(from + 512 * k + b1);
                    b[3 * k + 2] = shared2(from + 512 * k + b2);
                }
                __syncwarp();
                tc_store_scales(mine + kMxPairScaleCols * q.s, a, b);
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (one_lane()) mbar_arrive_first(ready + 8 * q.s);
            }
        }
    }
    __syncwarp();
    if (warp < 8) {
        const uint32_t quarter = warp & 3u, half = warp >> 2;
        constexpr uint32_t kSlabs = kMxPairN / 64;
        const uint32_t slabs = smem + S * kMxPairStageBytes + warp * SLABS * 4096;
        float* buf = reinterpret_cast<float*>(smem_raw + (slabs - smem_u32(smem_raw)));
        MxRing<2> u;        // places of sums
        MxRing<SLABS> w, l; // slabs worked on, slabs whose old values are asked for
        for (uint32_t tile = pair; tile < all_tiles && !wait.failed(); tile += pairs, u.next()) {
            const MxPairTile t(p, tile);
            const uint32_t sums_at = tmem + (quarter * 32 << 16) + u.s * kMxPairN + half * (kMxPairN / 2);
            const MxOutput o(p, t.n, t.row + rank * kMxTile + quarter * 32, t.col + half * (kMxPairN / 2), kMxPairN / 2, lane);
            const int row = (int)(t.row + rank * kMxTile + quarter * 32), col = (int)(t.col + half * (kMxPairN / 2));
            const uint32_t mine = by_tma && o.rows ? (o.cols + 31) / 32 : 0u; // slabs by TMA
            auto ask = [&](uint32_t slab) { // for a slab's old values, in a place whose last store has been read
                if (lane == 0) {
                    tma_stores_read<0>();
                    mbar_expect(old + 8 * (SLABS * warp + l.s), 4096);
                    tma_load_3d(slabs + 4096 * l.s, &map_out, col + 32 * (int)slab, row, (int)t.n, old + 8 * (SLABS * warp + l.s));
                }
                l.next();
            };
            if (p.beta != 0.f) {
#pragma unroll
                for (uint32_t i = 0; i < SLABS; ++i)
                    if (i < mine) ask(i);
            }
            if (!mbar_wait(done + 8 * u.s, u.parity, whole) || wait.failed()) break;
            __syncwarp();
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
            for (uint32_t slab = 0; slab < kSlabs; ++slab) {
                uint32_t sums[32];
                tc_load32(sums, sums_at + 32 * slab);
                if (slab == kSlabs - 1) { // the sums' place is free again
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (one_lane()) mbar_arrive_first(drained + 8 * u.s);
                }
                if (!by_tma) {
                    float was[32];
                    o.fetch(slab, was);
                    o.put(slab, sums, was, buf);
                }
                if (slab >= mine) continue;
                // sixteen bytes c of row r lie at c ^ (r % 8): no two of eight lanes meet in a bank
                const uint32_t at = slabs + 4096 * w.s + lane * 128;
                if (p.beta != 0.f) {
                    if (!mbar_wait(old + 8 * (SLABS * warp + w.s), w.parity, wait)) break;
                } else {
                    if (lane == 0) tma_stores_read<SLABS - 1>(); // the other places' stores may still be under way
                }
                __syncwarp();
#pragma unroll
                for (uint32_t c = 0; c < 8; ++c) {
                    const uint32_t place = at + ((c ^ (lane & 7u)) << 4);
                    float4 was = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (p.beta != 0.f) {
                        const uint4 x = shared4(place);
                        was = make_float4(__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w));
                    }
                    asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(place), "f"(o.update(sums[4 * c], was.x)), "f"(o.update(sums[4 * c + 1], was.y)),
                                 "f"(o.update(sums[4 * c + 2], was.z)), "f"(o.update(sums[4 * c + 3], was.w)) : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) tma_store_3d(&map_out, col + 32 * (int)slab, row, (int)t.n, slabs + 4096 * w.s);
                w.next();
                if (p.beta != 0.f && slab + SLABS < mine) ask(slab + SLABS);
            }
        }
        if (p.beta != 0.f) { // (after a failure: values asked for and not waited for)
            const long long began = clock64();
            for (; w.s != l.s || w.parity != l.parity; w.next())
                while (!mbar_try(old + 8 * (SLABS * warp + w.s), w.parity) && clock64() - began < kMxWaitClocks) {}
        }
        if (by_tma && lane == 0) tma_stores_done();
        __syncwarp();
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncthreads();
    if (s_failed) { // what was issued still writes to the pair's shared and tensor memory
        if (threadIdx.x == 0) mx_report(p.status);
        const long long began = clock64();
        if (warp == 12 && lane == 0 && rank == 0) // (the second CTA may be S stages ahead; a stage that only one has issued does not end, but its copies do within the limit)
            for (uint32_t i = it > S ? it - S : 0; i < it + S && !p.withhold; ++i)
                while (!mbar_try(codes + 8 * (i % S), (i / S) & 1u) && clock64() - began < kMxWaitClocks) {}
        if (warp == 14 && lane == 0)
            for (uint32_t i = it > S ? it - S : 0; i < it; ++i)
                while (!mbar_try(full + 8 * (i % S), (i / S) & 1u) && clock64() - began < kMxWaitClocks) {}
        if (warp == 13 && lane == 0 && rank == 0)
            while (!mbar_try(quit, 0) && clock64() - began < kMxWaitClocks) {}
        __syncwarp();
    }
    cluster_sync(); // neither CTA's memory goes before both are through with it
    if (warp == 13) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

} // namespace kimad
