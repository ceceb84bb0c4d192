// Microscaled 4-bit floats ("mx4"): the quantising compressor beside TopK, its receiving side, and matrices as operands of products.
//
// Block: 32 consecutive values of a layer (or of a line of an operand), the last one of it filled up with zeros.  With E the exponent field of
// the largest magnitude, the scale's byte is s = max(E - 2, 0) and its value 2^(s - 127); the values are rounded to the nearest multiple
// that E2M1 has (0, .5, 1, 1.5, 2, 3, 4, 6; ties to the even code) and end at 6 scales.  Multiplying by a power of two is exact here: the inverse
// scale is a normal number for every s in use, and what falls below the binary32 range then rounds to code 0 as it would have.
// A block with Inf or NaN has s = 255 and codes 0.
//   k_mx4_step       d = grad - g, C(d), g += C(d), ||d - C(d)||^2 (Eq. 4, Eq. 6 with this compressor)
//   k_mx4_stats      the layers' errors and the workers' records, where the pass does not see to them
//   k_mx4_apply      u^_m += C_m for every sender, and the model step (Algorithm 1, server lines)
//   k_mx4_read       a message as dense values
//   k_mx4_quantize_rows / _cols, k_mx4_dequantize_rows / _cols   operands (kimad_mx4_product.cuh multiplies them)
// All of them stream HBM once.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "kimad_kernels.cuh"

namespace kimad {

constexpr uint32_t kMxBlock = 32;   // values that share a scale
constexpr uint32_t kMxAbsent = 255; // scale byte of a block with Inf or NaN
constexpr uint32_t kMxPieces = 16;  // CTAs of a chunk at most
constexpr uint32_t kMxPer = 8;      // values of a lane: a warp has eight blocks in hand, four lanes each
constexpr uint32_t kMxGroup = 32 * kMxPer / kMxBlock, kMxGroupElems = 32 * kMxPer;
constexpr int kMxWarps = kThreads / 32;

struct __align__(16) MxPartial { // of a CTA of k_mx4_step
    double err;
    uint32_t absent, _pad;
};

// ---- One element of any type, and eight of them (32-byte aligned binary32, 16-byte aligned 16-bit types).
__device__ __forceinline__ float mx_float(float v) { return v; }
__device__ __forceinline__ float mx_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float mx_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T mx_make(float v);
template <> __device__ __forceinline__ float mx_make<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 mx_make<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half mx_make<__half>(float v) { return __float2half_rn(v); }

__device__ __forceinline__ void mx_load8(const float* p, float (&v)[8]) {
    asm volatile("ld.global.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "l"(p));
}
__device__ __forceinline__ void mx_load8(const __nv_bfloat16* p, float (&v)[8]) {
    const uint4 x = __ldcs(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void mx_load8(const __half* p, float (&v)[8]) {
    const uint4 x = __ldcs(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void mx_store8(float* p, const float (&v)[8]) {
    asm volatile("st.global.v8.f32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]),
                 "l"(p) : "memory");
}
__device__ __forceinline__ uint32_t mx_bf16x2(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void mx_store8(__nv_bfloat16* p, const float (&v)[8]) {
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(mx_bf16x2(v[0], v[1]), mx_bf16x2(v[2], v[3]), mx_bf16x2(v[4], v[5]), mx_bf16x2(v[6], v[7])));
}
template <typename T> __device__ __forceinline__ bool mx_aligned8(const T* p) { return reinterpret_cast<uintptr_t>(p) % (8 * sizeof(T)) == 0; }

// ---- Scales.  Byte of a block whose largest magnitude is `top` (NaN counts as larger than Inf), its inverse and its value (0 where the block is absent).
__device__ __forceinline__ float mx_max(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint32_t mx_byte(float top) {
    const uint32_t e = __float_as_uint(top) >> 23; // top has no sign
    return e >= 255u ? kMxAbsent : (e > 2u ? e - 2u : 0u);
}
__device__ __forceinline__ float mx_inverse(uint32_t byte) { return byte == kMxAbsent ? 0.f : __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ float mx_scale(uint32_t byte) { return byte == kMxAbsent ? 0.f : __uint_as_float(byte ? byte << 23 : 1u << 22); } // byte 0: 2^-127

// ---- Codes.  Eight scaled values as a word, the first one lowest, and back.
__device__ __forceinline__ uint32_t mx_codes8(const float (&r)[8]) {
    uint32_t w;
    asm("{\n.reg .b8 b0, b1, b2, b3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\ncvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\ncvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
        "mov.b32 %0, {b0, b1, b2, b3};\n}" : "=r"(w) : "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]));
    return w;
}
__device__ __forceinline__ void mx_values8(uint32_t w, float (&v)[8]) {
    uint32_t h[4];
    asm("{\n.reg .b8 b0, b1, b2, b3;\nmov.b32 {b0, b1, b2, b3}, %4;\n"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\ncvt.rn.f16x2.e2m1x2 %1, b1;\ncvt.rn.f16x2.e2m1x2 %2, b2;\ncvt.rn.f16x2.e2m1x2 %3, b3;\n}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

// Eight consecutive values of a lane, four lanes to a block: their codes, and the block's scale byte in all four lanes.
__device__ __forceinline__ uint32_t mx_quantize8(const float (&d)[8], uint32_t& byte) {
    float top = mx_max(mx_max(mx_max(fabsf(d[0]), fabsf(d[1])), mx_max(fabsf(d[2]), fabsf(d[3]))), mx_max(mx_max(fabsf(d[4]), fabsf(d[5])), mx_max(fabsf(d[6]), fabsf(d[7]))));
    top = mx_max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = mx_max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    byte = mx_byte(top);
    const float inv = mx_inverse(byte);
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = __fmul_rn(d[i], inv);
    const uint32_t word = mx_codes8(r);
    return byte == kMxAbsent ? 0u : word;
}

// ---- 256 consecutive elements in a warp.  In a lane's eight, WHOLE: elements 8 lane .. 8 lane + 7, by one vector access (aligned, none missing); otherwise
// elements lane + 32 j, j = 0 .. 7, one by one (any alignment, the first `lim` of the 256): lines of consecutive elements either way.
// Codes are made and read in the first order; the second one changes to it and back through 1 KB of shared memory per warp.
template <bool WHOLE, typename T> __device__ __forceinline__ void mx_get(const T* p, uint32_t lim, uint32_t lane, float (&v)[8]) {
    if (WHOLE) mx_load8(p + lane * 8, v);
    else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
            const T x = lane + 32 * j < lim ? p[lane + 32 * j] : mx_make<T>(0.f);
            v[j] = mx_float(x);
        }
    }
}
template <bool WHOLE, typename T> __device__ __forceinline__ void mx_put(T* p, uint32_t lim, uint32_t lane, const float (&v)[8], uint32_t gone) {
    if (WHOLE) {
        if (!(gone >> lane & 1u)) mx_store8(p + lane * 8, v);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j)
            if (lane + 32 * j < lim && !(gone >> (4 * j) & 1u)) p[lane + 32 * j] = mx_make<T>(v[j]);
    }
}
template <bool WHOLE> __device__ __forceinline__ void mx_to_blocks(float (&v)[8], float* buf, uint32_t lane) {
    if (WHOLE) return;
    __syncwarp();
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) buf[lane + 32 * j] = v[j];
    __syncwarp();
    const float4 a = reinterpret_cast<const float4*>(buf)[2 * lane], b = reinterpret_cast<const float4*>(buf)[2 * lane + 1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
template <bool WHOLE> __device__ __forceinline__ void mx_from_blocks(float (&v)[8], float* buf, uint32_t lane) {
    if (WHOLE) return;
    __syncwarp();
    reinterpret_cast<float4*>(buf)[2 * lane] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(buf)[2 * lane + 1] = make_float4(v[4], v[5], v[6], v[7]);
    __syncwarp();
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) v[j] = buf[lane + 32 * j];
}

// The blocks of a chunk: those that start inside it.  They may reach into the layer's next chunk.
struct MxSpan {
    uint64_t base;         // flat index of the first block's first element
    uint64_t first;        // the first block's place in the worker's message
    uint32_t blocks, left; // elements from base on that are the layer's
    __device__ __forceinline__ MxSpan(const Chunk& ch, const LayerDesc& ld) {
        const uint64_t b0 = (ch.begin - ld.begin + kMxBlock - 1) / kMxBlock, b1 = (ch.end - ld.begin + kMxBlock - 1) / kMxBlock;
        base = ld.begin + b0 * kMxBlock;
        first = ch.block;
        blocks = (uint32_t)(b1 - b0);
        left = blocks ? (uint32_t)min(ld.n - b0 * kMxBlock, (uint64_t)blocks * kMxBlock) : 0u;
    }
};

// Where a worker's message lies.
struct MxMessage {
    uint8_t *codes, *scales;
    uint64_t code_bytes, scale_bytes; // of a worker
    __device__ __forceinline__ uint32_t* words(uint32_t w, uint64_t first) const { return reinterpret_cast<uint32_t*>(codes + (size_t)w * code_bytes) + first * 4; }
    __device__ __forceinline__ uint8_t* bytes(uint32_t w, uint64_t first) const { return scales + (size_t)w * scale_bytes + first; }
    __device__ __forceinline__ bool holds(uint64_t first, uint32_t blocks) const { return (first + blocks) * 16 <= code_bytes && first + blocks <= scale_bytes; }
};

// Eight blocks of a pass: values, message, estimator.  `blocks` of them are there.
template <bool WHOLE, typename T>
__device__ __forceinline__ void mx_step_group(const T* g, float* st, uint32_t lim, uint32_t lane, uint32_t blocks, uint32_t* words, uint8_t* bytes, float* buf,
                                              double& err, uint32_t& absent) {
    float d[8], s[8], v[8];
    mx_get<WHOLE>(st, lim, lane, s);
    mx_get<WHOLE>(g, lim, lane, d);
#pragma unroll
    for (int j = 0; j < 8; ++j) d[j] = __fsub_rn(d[j], s[j]);
    mx_to_blocks<WHOLE>(d, buf, lane);
    uint32_t byte;
    const uint32_t word = mx_quantize8(d, byte);
    mx_values8(word, v);
    const float x = mx_scale(byte);
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        v[j] = __fmul_rn(v[j], x);
        const double off = (double)__fsub_rn(d[j], v[j]);
        sum = fma(off, off, sum);
    }
    const uint32_t gone = __ballot_sync(0xffffffffu, byte == kMxAbsent);
    if (byte != kMxAbsent) err += sum;
    absent += __popc(gone) / 4u;
    mx_from_blocks<WHOLE>(v, buf, lane);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __fadd_rn(s[j], v[j]);
    mx_put<WHOLE>(st, lim, lane, v, gone);
    if (WHOLE || lane / 4 < blocks) {
        words[lane] = word;
        if (lane % 4 == 0) bytes[lane / 4] = (uint8_t)byte;
    }
}

// What becomes of the CTAs' sums: the layers' errors and the worker's record.
struct MxStats {
    MxPartial* partial; // [W][CTAs of a worker]
    uint32_t* arrived;  // [W] CTAs that have left their sums, zero before and after; null where they are not counted
    float* err;
    kimad_stats* stats;
    uint64_t n, message_bytes;
    uint32_t L, check_finite;
};

// By one CTA for a worker.  The sums of a layer of few are added up by a thread, those of one of many by a warp, and by the CTA where a warp would
// take long; the order depends on the layers only.  A layer with an absent block has an infinite error, as its difference has.
template <uint32_t THREADS>
__device__ __forceinline__ void mx_stats(const MxStats& st, const LayerDesc* layers, uint32_t w, uint32_t ctas, uint32_t log_pieces, double* s_err, uint32_t* s_absent) {
    constexpr uint32_t WARPS = THREADS / 32;
    constexpr uint32_t kFew = 8, kMany = 256;
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const MxPartial* mine = st.partial + (size_t)w * ctas;
    double total = 0.0;
    uint32_t absent = 0;
    auto add = [&](const LayerDesc& ld, uint32_t from, uint32_t step, double& sum, uint32_t& gone) {
        const uint4* at = reinterpret_cast<const uint4*>(mine + ((size_t)ld.first_chunk << log_pieces));
        const uint32_t count = ld.n_chunks << log_pieces;
        sum = 0.0;
        gone = 0;
#pragma unroll 4
        for (uint32_t i = from; i < count; i += step) {
            const uint4 p = __ldcg(at + i); // written by other CTAs of this kernel
            sum += __hiloint2double((int)p.y, (int)p.x);
            gone += p.z;
        }
    };
    auto over_warp = [&](double& sum, uint32_t& gone) {
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, o);
            gone += __shfl_xor_sync(0xffffffffu, gone, o);
        }
    };
    auto over_cta = [&](double& sum, uint32_t& gone) { // the result is thread 0's
        over_warp(sum, gone);
        __syncthreads();
        if (lane == 0) { s_err[warp] = sum; s_absent[warp] = gone; }
        __syncthreads();
        if (threadIdx.x == 0)
            for (uint32_t i = 1; i < WARPS; ++i) { sum += s_err[i]; gone += s_absent[i]; }
    };
    auto done = [&](uint32_t l, double sum, uint32_t gone) {
        if (gone) sum = (double)__int_as_float(0x7f800000);
        st.err[(size_t)w * st.L + l] = (float)sum;
        total += sum;
        absent += gone;
    };
    uint32_t many = 0;
    for (uint32_t l = threadIdx.x; l < st.L; l += THREADS) {
        const LayerDesc ld = layers[l];
        const uint32_t count = ld.n_chunks << log_pieces;
        many += count > kMany;
        if (count > kFew) continue;
        double sum;
        uint32_t gone;
        add(ld, 0, 1, sum, gone);
        done(l, sum, gone);
    }
    for (uint32_t l = warp; l < st.L; l += WARPS) {
        const LayerDesc ld = layers[l];
        const uint32_t count = ld.n_chunks << log_pieces;
        if (count <= kFew || count > kMany) continue;
        double sum;
        uint32_t gone;
        add(ld, lane, 32, sum, gone);
        over_warp(sum, gone);
        if (lane == 0) done(l, sum, gone);
    }
    if (__syncthreads_or(many))
        for (uint32_t l = 0; l < st.L; ++l) {
            const LayerDesc ld = layers[l];
            if (ld.n_chunks << log_pieces <= kMany) continue;
            double sum;
            uint32_t gone;
            add(ld, threadIdx.x, THREADS, sum, gone);
            over_cta(sum, gone);
            if (threadIdx.x == 0) done(l, sum, gone);
        }
    over_cta(total, absent);
    if (threadIdx.x == 0) {
        kimad_stats s{};
        s.used_bytes = st.message_bytes;
        s.n_selected = st.n;
        s.total_err = (float)total;
        s.status = absent && st.check_finite ? KIMAD_ERR_NONFINITE : KIMAD_OK;
        st.stats[w] = s;
    }
}

// Where the CTAs are few, the last one of a worker does that: the pass of a small model then is one launch (0.10 M elements: 4.5 us of the host's time instead of
// 6.3).  Where they are many, a kernel of its own behind them: their arrivals and the smaller CTA cost more there (124 M elements in odd layers 285 us instead of 277).
constexpr uint32_t kMxStatsThreads = 1024;
__global__ void __launch_bounds__(kMxStatsThreads)
k_mx4_stats(MxStats st, const LayerDesc* __restrict__ layers, uint32_t ctas, uint32_t log_pieces) {
    pdl_wait();
    __shared__ double s_err[kMxStatsThreads / 32];
    __shared__ uint32_t s_absent[kMxStatsThreads / 32];
    mx_stats<kMxStatsThreads>(st, layers, blockIdx.x, ctas, log_pieces, s_err, s_absent);
}

// One CTA per chunk, or per piece of one (1 << log_pieces of them) where the chunks are few; a warp takes eight blocks at a time.  Bound by HBM: 12.53
// bytes per element with f32 gradients, 10.53 with 16-bit ones.  The difference d - C(d) is exact in binary32 (C(d) is zero or a multiple of half
// a scale beside d), its squares are added in binary64: per lane, per CTA, per layer, always in the same order.
// (A lane per element of a block, with the block's largest magnitude by a reduction over the warp, needs no vectors and no alignment but works
// every scale out 32 times, 55 instructions per element: 4 x 124 M elements with bf16 gradients 1170 us, 839 this way.)
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_mx4_step(const T* __restrict__ grads, float* __restrict__ state, uint64_t stride, const Chunk* __restrict__ chunks,
           const LayerDesc* __restrict__ layers, uint32_t log_pieces, MxMessage msg, MxStats st) {
    pdl_wait();
    __shared__ __align__(16) float s_buf[kMxWarps][kMxGroupElems];
    __shared__ double s_err[kMxWarps];
    __shared__ uint32_t s_absent[kMxWarps], s_last;
    const uint32_t w = blockIdx.y, f = blockIdx.x >> log_pieces, pieces = 1u << log_pieces, piece = blockIdx.x & (pieces - 1u);
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Chunk ch = chunks[f];
    const MxSpan sp(ch, layers[ch.layer]);
    const T* g = grads + (size_t)w * stride + sp.base;
    float* at = state + (size_t)w * stride + sp.base;
    uint32_t* words = msg.words(w, sp.first);
    uint8_t* bytes = msg.bytes(w, sp.first);
    const bool aligned = mx_aligned8(g) && mx_aligned8(at);
    double err = 0.0;
    uint32_t absent = 0;
    for (uint32_t b = (piece * kMxWarps + warp) * kMxGroup; b < sp.blocks; b += pieces * kMxWarps * kMxGroup) {
        const uint32_t e = b * kMxBlock, lim = min(sp.left - e, kMxGroupElems), blocks = min(sp.blocks - b, kMxGroup);
        if (!KIMAD_CHECK(msg.holds(sp.first + b, blocks), 8)) break;
        if (aligned && lim == kMxGroupElems) mx_step_group<true>(g + e, at + e, lim, lane, blocks, words + b * 4, bytes + b, nullptr, err, absent);
        else mx_step_group<false>(g + e, at + e, lim, lane, blocks, words + b * 4, bytes + b, s_buf[warp], err, absent);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) err += __shfl_xor_sync(0xffffffffu, err, o);
    if (lane == 0) { s_err[warp] = err; s_absent[warp] = absent; }
    __syncthreads();
    if (threadIdx.x == 0) {
        MxPartial p{0.0, 0, 0};
        for (int i = 0; i < kMxWarps; ++i) { p.err += s_err[i]; p.absent += s_absent[i]; }
        st.partial[(size_t)w * gridDim.x + blockIdx.x] = p;
        if (st.arrived) {
            __threadfence();
            s_last = atomicInc(st.arrived + w, gridDim.x - 1) == gridDim.x - 1; // back to zero with the last one
            __threadfence();
        }
    }
    if (!st.arrived) return;
    __syncthreads();
    if (s_last) mx_stats<kThreads>(st, layers, w, gridDim.x, log_pieces, s_err, s_absent);
}

// Eight blocks of a message in a warp: a lane's eight values (0 where the block is absent); the lanes of absent blocks come back as a mask.
__device__ __forceinline__ void mx_fetch(const uint32_t* words, const uint8_t* bytes, uint32_t blocks, uint32_t lane, uint32_t& word, uint32_t& byte) {
    word = lane / 4 < blocks ? __ldcs(words + lane) : 0u;
    byte = lane / 4 < blocks ? (uint32_t)__ldcs(bytes + lane / 4) : 0u;
}
__device__ __forceinline__ uint32_t mx_decode(uint32_t word, uint32_t byte, float (&v)[8]) {
    mx_values8(word, v);
    const float x = mx_scale(byte);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = byte == kMxAbsent ? 0.f : __fmul_rn(v[j], x);
    return __ballot_sync(0xffffffffu, byte == kMxAbsent);
}

struct MxWeights { float w[KIMAD_MAX_AGG_WORKERS]; };

// Eight blocks of the senders m_first .. m_end - 1, and of the model; the loads of two senders are in flight at a time.
template <bool WHOLE, bool MODEL>
__device__ __forceinline__ void mx_apply_group(const MxMessage& msg, uint64_t first, float* est, uint64_t stride, float* x, uint32_t lim, uint32_t lane,
                                               uint32_t blocks, uint32_t m_first, uint32_t m_end, const MxWeights& wt, float gamma, float* buf) {
    constexpr uint32_t U = MODEL ? 2 : 1;
    float acc[8] = {}, xv[8];
    if (MODEL) mx_get<WHOLE>(x, lim, lane, xv);
    for (uint32_t m0 = m_first; m0 < m_end; m0 += U) {
        uint32_t word[U], byte[U];
        float s[U][8];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            const uint32_t m = min(m0 + u, m_end - 1u);
            mx_fetch(msg.words(m, first), msg.bytes(m, first), blocks, lane, word[u], byte[u]);
            mx_get<WHOLE>(est + (size_t)m * stride, m0 + u < m_end ? lim : 0u, lane, s[u]);
        }
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            if (m0 + u >= m_end) break;
            float v[8];
            const uint32_t gone = mx_decode(word[u], byte[u], v);
            mx_from_blocks<WHOLE>(v, buf, lane);
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) s[u][j] = gone >> (WHOLE ? lane : 4 * j) & 1u ? s[u][j] : __fadd_rn(s[u][j], v[j]);
            mx_put<WHOLE>(est + (size_t)(m0 + u) * stride, lim, lane, s[u], gone);
            if (MODEL) {
                const float wm = wt.w[m0 + u];
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) acc[j] = __fadd_rn(acc[j], __fmul_rn(wm, s[u][j]));
            }
        }
    }
    if (MODEL) {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) xv[j] = __fsub_rn(xv[j], __fmul_rn(gamma, acc[j]));
        mx_put<WHOLE>(x, lim, lane, xv, 0u);
    }
}

// Same cut of the work as k_mx4_step.  Without the model a CTA has one sender (blockIdx.y); with it, all of them: an estimator's entry is then read
// and written once, and the model step (the order of k_aggregate's operations) costs the model's own 8 bytes instead of another
// pass over all estimators.  An absent block leaves its estimator as it is.
template <bool MODEL>
__global__ void __launch_bounds__(kThreads)
k_mx4_apply(MxMessage msg, const Chunk* __restrict__ chunks, const LayerDesc* __restrict__ layers, uint32_t log_pieces, float* __restrict__ est,
            uint64_t stride, uint32_t W, float* __restrict__ x, const __grid_constant__ MxWeights wt, float gamma) {
    pdl_wait();
    __shared__ __align__(16) float s_buf[kMxWarps][kMxGroupElems];
    const uint32_t f = blockIdx.x >> log_pieces, pieces = 1u << log_pieces, piece = blockIdx.x & (pieces - 1u);
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Chunk ch = chunks[f];
    const MxSpan sp(ch, layers[ch.layer]);
    const uint32_t m_first = MODEL ? 0u : blockIdx.y, m_end = MODEL ? W : blockIdx.y + 1u;
    float *at = est + sp.base, *xa = MODEL ? x + sp.base : nullptr;
    const bool aligned = mx_aligned8(at + (size_t)m_first * stride) && (!MODEL || (mx_aligned8(xa) && (W == 1 || stride % 8 == 0)));
    for (uint32_t b = (piece * kMxWarps + warp) * kMxGroup; b < sp.blocks; b += pieces * kMxWarps * kMxGroup) {
        const uint32_t e = b * kMxBlock, lim = min(sp.left - e, kMxGroupElems), blocks = min(sp.blocks - b, kMxGroup);
        if (!KIMAD_CHECK(msg.holds(sp.first + b, blocks), 8)) break;
        if (aligned && lim == kMxGroupElems)
            mx_apply_group<true, MODEL>(msg, sp.first + b, at + e, stride, xa + (MODEL ? e : 0), lim, lane, blocks, m_first, m_end, wt, gamma, nullptr);
        else mx_apply_group<false, MODEL>(msg, sp.first + b, at + e, stride, xa + (MODEL ? e : 0), lim, lane, blocks, m_first, m_end, wt, gamma, s_buf[warp]);
    }
}

// C(d) as dense values (0 where a block is absent).  bfloat16 holds every one of them exactly: two significant bits and bfloat16's exponents.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_mx4_read(MxMessage msg, const Chunk* __restrict__ chunks, const LayerDesc* __restrict__ layers, uint32_t log_pieces, T* __restrict__ out, uint64_t stride) {
    pdl_wait();
    __shared__ __align__(16) float s_buf[kMxWarps][kMxGroupElems];
    const uint32_t w = blockIdx.y, f = blockIdx.x >> log_pieces, pieces = 1u << log_pieces, piece = blockIdx.x & (pieces - 1u);
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Chunk ch = chunks[f];
    const MxSpan sp(ch, layers[ch.layer]);
    T* o = out + (size_t)w * stride + sp.base;
    const uint32_t* words = msg.words(w, sp.first);
    const uint8_t* bytes = msg.bytes(w, sp.first);
    const bool aligned = mx_aligned8(o);
    constexpr uint32_t U = 4; // groups under way
    const uint32_t step = pieces * kMxWarps * kMxGroup;
    for (uint32_t b0 = (piece * kMxWarps + warp) * kMxGroup; b0 < sp.blocks; b0 += U * step) {
        uint32_t word[U], byte[U];
        if (!KIMAD_CHECK(msg.holds(sp.first, sp.blocks), 8)) break;
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            const uint32_t b = b0 + u * step;
            mx_fetch(words + b * 4, bytes + b, b < sp.blocks ? sp.blocks - b : 0u, lane, word[u], byte[u]);
        }
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            const uint32_t b = b0 + u * step, e = b * kMxBlock;
            if (b >= sp.blocks) break;
            const uint32_t lim = min(sp.left - e, kMxGroupElems);
            float v[8];
            mx_decode(word[u], byte[u], v);
            if (aligned && lim == kMxGroupElems) mx_put<true>(o + e, lim, lane, v, 0u);
            else {
                mx_from_blocks<false>(v, s_buf[warp], lane);
                mx_put<false>(o + e, lim, lane, v, 0u);
            }
        }
    }
}

// ---- Operands.  `lines` lines of `length` values with blocks along a line: codes [batch][lines][16 * blocks] bytes, scales in tiles of 128 lines by
// 4 blocks, [batch][lines / 128][blocks / 4][512] (rounded up): line r and block b of a tile at byte (r % 32) * 16 + r / 32 * 4 + b, the
// order in which the tensor cores take them (kimad_mx4_product.cuh).  Scales of lines and blocks that are not there are 0.
constexpr uint32_t kMxTile = 128;
struct MxOperand {
    uint32_t lines, length, blocks, line_tiles, block_tiles;
    KIMAD_HD MxOperand(uint32_t lines_, uint32_t length_)
        : lines(lines_), length(length_), blocks((length_ + kMxBlock - 1) / kMxBlock), line_tiles((lines_ + kMxTile - 1) / kMxTile),
          block_tiles((blocks + 3) / 4) {}
    KIMAD_HD uint64_t code_bytes() const { return (uint64_t)lines * blocks * 16; }
    KIMAD_HD uint64_t scale_bytes() const { return (uint64_t)line_tiles * block_tiles * 512; }
    __device__ __forceinline__ bool holds(uint32_t line, uint32_t block) const {
        return ((uint64_t)line * blocks + block + 1) * 16 <= code_bytes() && scale_word(line, block / 4) * 4 + block % 4 < scale_bytes();
    }
    // the four scales of a line in a tile of blocks, as a word
    KIMAD_HD uint64_t scale_word(uint32_t line, uint32_t tile) const {
        return ((uint64_t)(line / kMxTile) * block_tiles + tile) * 128 + (line % 32) * 4 + line % kMxTile / 32;
    }
};

// Blocks along the contiguous axis: a warp has 256 values of a line in hand at a time, as in a message; a CTA eight lines by kMxRowGroups of these.
// Lines that fill the last tile up get their scales of 0.
constexpr uint32_t kMxRowGroups = 4;
struct MxRowCuts { // CTAs of a matrix: groups of eight lines by pieces of a line
    uint32_t groups, line_sets, pieces;
    KIMAD_HD MxRowCuts(const MxOperand& op)
        : groups((op.blocks + kMxGroup - 1) / kMxGroup), line_sets(op.line_tiles * (kMxTile / 8)), pieces((groups + kMxRowGroups - 1) / kMxRowGroups) {}
    KIMAD_HD uint64_t ctas() const { return (uint64_t)line_sets * pieces; }
};
static_assert(kMxWarps == 8, "a warp for each of eight lines");

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_mx4_quantize_rows(const T* __restrict__ x, uint64_t ld, uint64_t batch_stride, MxOperand op, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    pdl_wait();
    __shared__ __align__(16) float s_buf[kMxWarps][kMxGroupElems];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const MxRowCuts cuts(op);
    const uint32_t piece = blockIdx.x % cuts.pieces, line = blockIdx.x / cuts.pieces % cuts.line_sets * 8 + warp;
    const uint64_t n = blockIdx.x / cuts.pieces / cuts.line_sets;
    const uint32_t b0 = piece * kMxRowGroups * kMxGroup, e0 = b0 * kMxBlock, left = line < op.lines ? op.length - e0 : 0u; // values of the line from e0 on
    const T* row = x + n * batch_stride + (uint64_t)min(line, op.lines - 1) * ld + e0;
    uint32_t* words = reinterpret_cast<uint32_t*>(codes) + ((n * op.lines + line) * op.blocks + b0) * 4;
    uint8_t* tiles = scales + n * op.scale_bytes();
    float v[kMxRowGroups][8]; // all under way at once
    if (mx_aligned8(row) && left >= kMxRowGroups * kMxGroupElems) {
#pragma unroll
        for (uint32_t i = 0; i < kMxRowGroups; ++i) mx_get<true>(row + i * kMxGroupElems, kMxGroupElems, lane, v[i]);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < kMxRowGroups; ++i) mx_get<false>(row + i * kMxGroupElems, left > i * kMxGroupElems ? left - i * kMxGroupElems : 0u, lane, v[i]);
#pragma unroll
        for (uint32_t i = 0; i < kMxRowGroups; ++i) mx_to_blocks<false>(v[i], s_buf[warp], lane);
    }
#pragma unroll
    for (uint32_t i = 0; i < kMxRowGroups; ++i) {
        const uint32_t own = b0 + i * kMxGroup + lane / 4;
        uint32_t byte;
        const uint32_t word = mx_quantize8(v[i], byte);
        if (line < op.lines && own < op.blocks && KIMAD_CHECK(op.holds(line, own), 9)) words[i * 32 + lane] = word;
        if (lane % 4 == 0 && own < op.block_tiles * 4) tiles[op.scale_word(line, own / 4) * 4 + own % 4] = (uint8_t)byte;
    }
}

// Blocks along the other axis, which transposes: a CTA takes 128 lines (columns of x) by 128 values (rows), a lane one block of each of two
// neighbouring columns.  Rows are read in whole lines and a block's values need no exchange between lanes; codes go through shared memory so that 64
// bytes of a line are written together.  Pairs of columns are read as one where they are aligned and the tile is whole.
// (One column per lane and 16-bit loads, 28 instructions per value: 8192 x 5632 bfloat16 values 133 us, 27 this way.  Lanes write and read their codes 128
// bytes apart, so that eight of them meet in four banks: half of the shared memory's cycles, here and on the way back, beside HBM's.)
template <typename T> struct MxPair;
template <> struct MxPair<float> {
    float2 v;
    __device__ __forceinline__ float lo() const { return v.x; }
    __device__ __forceinline__ float hi() const { return v.y; }
};
template <> struct MxPair<__nv_bfloat16> {
    uint32_t v;
    __device__ __forceinline__ float lo() const { return __uint_as_float(v << 16); }
    __device__ __forceinline__ float hi() const { return __uint_as_float(v & 0xffff0000u); }
};
template <> struct MxPair<__half> {
    uint32_t v;
    __device__ __forceinline__ float lo() const { return __low2float(*reinterpret_cast<const __half2*>(&v)); }
    __device__ __forceinline__ float hi() const { return __high2float(*reinterpret_cast<const __half2*>(&v)); }
};
__device__ __forceinline__ MxPair<float> mx_pair(float lo, float hi) { return {make_float2(lo, hi)}; }
__device__ __forceinline__ MxPair<__nv_bfloat16> mx_pair(__nv_bfloat16 lo, __nv_bfloat16 hi) { return {__bfloat16_as_ushort(lo) | (uint32_t)__bfloat16_as_ushort(hi) << 16}; }
__device__ __forceinline__ MxPair<__half> mx_pair(__half lo, __half hi) { return {__half_as_ushort(lo) | (uint32_t)__half_as_ushort(hi) << 16}; }
// The largest magnitudes of both columns: of 16-bit types as two integers in a word, whose order is that of the magnitudes with NaN on top.
struct MxTops {
    float lo = 0.f, hi = 0.f;
    __device__ __forceinline__ void see(const MxPair<float>& p) { lo = mx_max(lo, fabsf(p.v.x)); hi = mx_max(hi, fabsf(p.v.y)); }
    template <typename T> __device__ __forceinline__ void done() {}
};
struct MxTops16 {
    uint32_t top = 0;
    float lo = 0.f, hi = 0.f;
    template <typename T> __device__ __forceinline__ void see(const MxPair<T>& p) { top = __vmaxu2(top, p.v & 0x7fff7fffu); }
    template <typename T> __device__ __forceinline__ void done() { const MxPair<T> p{top}; lo = p.lo(); hi = p.hi(); }
};

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_mx4_quantize_cols(const T* __restrict__ x, uint64_t ld, uint64_t batch_stride, MxOperand op, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    pdl_wait();
    __shared__ uint4 s_codes[kMxTile][4];
    __shared__ __align__(4) uint8_t s_scales[512];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t lt = blockIdx.x % op.line_tiles, bt = blockIdx.x / op.line_tiles % op.block_tiles;
    const uint64_t n = blockIdx.x / op.line_tiles / op.block_tiles;
    const uint32_t in_line = (warp & 1u) * 64 + lane * 2, line = lt * kMxTile + in_line, q = warp >> 1, row0 = (bt * 4 + q) * kMxBlock;
    const T* from = x + n * batch_stride + (uint64_t)row0 * ld + line;
    MxPair<T> v[kMxBlock];
    if ((lt + 1) * kMxTile <= op.lines && (bt + 1) * kMxTile <= op.length && ld % 2 == 0 && reinterpret_cast<uintptr_t>(from) % (2 * sizeof(T)) == 0) {
#pragma unroll
        for (uint32_t i = 0; i < kMxBlock; ++i) v[i].v = __ldcs(reinterpret_cast<const decltype(v[i].v)*>(from + i * ld));
    } else {
#pragma unroll
        for (uint32_t i = 0; i < kMxBlock; ++i) {
            const T lo = line < op.lines && row0 + i < op.length ? from[i * ld] : mx_make<T>(0.f);
            const T hi = line + 1 < op.lines && row0 + i < op.length ? from[i * ld + 1] : mx_make<T>(0.f);
            v[i] = mx_pair(lo, hi);
        }
    }
    std::conditional_t<sizeof(T) == 2, MxTops16, MxTops> top;
#pragma unroll
    for (uint32_t i = 0; i < kMxBlock; ++i) top.see(v[i]);
    top.template done<T>();
#pragma unroll
    for (uint32_t u = 0; u < 2; ++u) {
        const uint32_t byte = mx_byte(u ? top.hi : top.lo);
        const float inv = mx_inverse(byte);
        uint32_t word[4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            float r[8];
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) r[j] = __fmul_rn(u ? v[8 * i + j].hi() : v[8 * i + j].lo(), inv);
            word[i] = mx_codes8(r);
            if (byte == kMxAbsent) word[i] = 0;
        }
        s_codes[in_line + u][q] = make_uint4(word[0], word[1], word[2], word[3]);
        s_scales[(in_line + u) % 32 * 16 + in_line / 32 * 4 + q] = (uint8_t)byte;
    }
    __syncthreads();
#pragma unroll
    for (uint32_t i = threadIdx.x; i < kMxTile * 4; i += kThreads) {
        const uint32_t out = lt * kMxTile + i / 4, block = bt * 4 + i % 4;
        if (out < op.lines && block < op.blocks && KIMAD_CHECK(op.holds(out, block), 9)) reinterpret_cast<uint4*>(codes)[(n * op.lines + out) * op.blocks + block] = s_codes[i / 4][i % 4];
    }
    if (threadIdx.x < 128)
        reinterpret_cast<uint32_t*>(scales)[((n * op.line_tiles + lt) * op.block_tiles + bt) * 128 + threadIdx.x] = reinterpret_cast<uint32_t*>(s_scales)[threadIdx.x];
}

// Back to values, both ways round.  A block that could not be quantised reads as NaN.
__device__ __forceinline__ float mx_operand_scale(uint32_t byte) { return byte == kMxAbsent ? __int_as_float(0x7fffffff) : mx_scale(byte); }

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_mx4_dequantize_rows(T* __restrict__ x, uint64_t ld, uint64_t batch_stride, MxOperand op, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales) {
    pdl_wait();
    __shared__ __align__(16) float s_buf[kMxWarps][kMxGroupElems];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const MxRowCuts cuts(op);
    const uint32_t piece = blockIdx.x % cuts.pieces, line = blockIdx.x / cuts.pieces % cuts.line_sets * 8 + warp;
    const uint64_t n = blockIdx.x / cuts.pieces / cuts.line_sets;
    if (line >= op.lines) return;
    const uint32_t b0 = piece * kMxRowGroups * kMxGroup, e0 = b0 * kMxBlock, left = op.length - e0;
    T* row = x + n * batch_stride + (uint64_t)line * ld + e0;
    const uint32_t* words = reinterpret_cast<const uint32_t*>(codes) + ((n * op.lines + line) * op.blocks + b0) * 4;
    const uint8_t* tiles = scales + n * op.scale_bytes();
    const bool aligned = mx_aligned8(row);
    uint32_t word[kMxRowGroups], byte[kMxRowGroups]; // all under way at once
#pragma unroll
    for (uint32_t i = 0; i < kMxRowGroups; ++i) {
        const uint32_t own = b0 + i * kMxGroup + lane / 4;
        const bool here = own < op.blocks && KIMAD_CHECK(op.holds(line, own), 9);
        word[i] = here ? __ldcs(words + i * 32 + lane) : 0u;
        byte[i] = here ? (uint32_t)tiles[op.scale_word(line, own / 4) * 4 + own % 4] : 0u;
    }
#pragma unroll
    for (uint32_t i = 0; i < kMxRowGroups; ++i) {
        const uint32_t e = i * kMxGroupElems;
        if (e >= left) break;
        const uint32_t lim = min(left - e, kMxGroupElems);
        const float scale = mx_operand_scale(byte[i]);
        float v[8];
        mx_values8(word[i], v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __fmul_rn(v[j], scale);
        if (aligned && lim == kMxGroupElems) mx_put<true>(row + e, lim, lane, v, 0u);
        else {
            mx_from_blocks<false>(v, s_buf[warp], lane);
            mx_put<false>(row + e, lim, lane, v, 0u);
        }
    }
}

__device__ __forceinline__ void mx_store2(float* p, float lo, float hi) { __stcs(reinterpret_cast<float2*>(p), make_float2(lo, hi)); }
__device__ __forceinline__ void mx_store2(__nv_bfloat16* p, float lo, float hi) { __stcs(reinterpret_cast<uint32_t*>(p), mx_bf16x2(lo, hi)); }

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_mx4_dequantize_cols(T* __restrict__ x, uint64_t ld, uint64_t batch_stride, MxOperand op, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales) {
    pdl_wait();
    __shared__ uint4 s_codes[kMxTile][4];
    __shared__ uint32_t s_scales[128];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t lt = blockIdx.x % op.line_tiles, bt = blockIdx.x / op.line_tiles % op.block_tiles;
    const uint64_t n = blockIdx.x / op.line_tiles / op.block_tiles;
#pragma unroll
    for (uint32_t i = threadIdx.x; i < kMxTile * 4; i += kThreads) {
        const uint32_t in = lt * kMxTile + i / 4, block = bt * 4 + i % 4;
        if (in < op.lines && block < op.blocks && KIMAD_CHECK(op.holds(in, block), 9)) s_codes[i / 4][i % 4] = __ldcs(reinterpret_cast<const uint4*>(codes) + (n * op.lines + in) * op.blocks + block);
    }
    if (threadIdx.x < 128) s_scales[threadIdx.x] = __ldcs(reinterpret_cast<const uint32_t*>(scales) + ((n * op.line_tiles + lt) * op.block_tiles + bt) * 128 + threadIdx.x);
    __syncthreads();
    const uint32_t in_line = (warp & 1u) * 64 + lane * 2, line = lt * kMxTile + in_line, q = warp >> 1, row0 = (bt * 4 + q) * kMxBlock;
    if (line >= op.lines || bt * 4 + q >= op.blocks) return;
    const uint4 c0 = s_codes[in_line][q], c1 = s_codes[in_line + 1][q]; // (the second one may be behind the last line: not stored then)
    const uint32_t w0[4] = {c0.x, c0.y, c0.z, c0.w}, w1[4] = {c1.x, c1.y, c1.z, c1.w};
    const float x0 = mx_operand_scale((s_scales[in_line % 32 * 4 + in_line / 32] >> (8 * q)) & 255u);
    const float x1 = mx_operand_scale((s_scales[in_line % 32 * 4 + 4 + in_line / 32] >> (8 * q)) & 255u);
    T* to = x + n * batch_stride + (uint64_t)row0 * ld + line;
    const bool two = (lt + 1) * kMxTile <= op.lines && (bt + 1) * kMxTile <= op.length && ld % 2 == 0 && reinterpret_cast<uintptr_t>(to) % (2 * sizeof(T)) == 0;
    if (two) {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            float v0[8], v1[8];
            mx_values8(w0[i], v0);
            mx_values8(w1[i], v1);
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j, to += ld) mx_store2(to, __fmul_rn(v0[j], x0), __fmul_rn(v1[j], x1));
        }
        return;
    }
    const uint32_t rows = min(op.length - row0, kMxBlock), rows1 = line + 1 < op.lines ? rows : 0u;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        float v0[8], v1[8];
        mx_values8(w0[i], v0);
        mx_values8(w1[i], v1);
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j, to += ld) {
            if (8 * i + j < rows) to[0] = mx_make<T>(__fmul_rn(v0[j], x0));
            if (8 * i + j < rows1) to[1] = mx_make<T>(__fmul_rn(v1[j], x1));
        }
    }
}

} // namespace kimad
