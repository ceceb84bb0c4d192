// Microscaled 4-bit floats ("mx4"): the quantising compressor beside TopK, its receiving side, and matrices as operands of products.
//
// Block: 32 consecutive values of a layer (or of a line of an operand), the last one of it filled up with zeros.  With E the exponent field of
// the largest magnitude, the scale's byte is s = max(E - 2, 0) and its value 2^(s - 127); the values are rounded to the nearest multiple
// that E2M1 has (0, .5, 1, 1.5, 2, 3, 4, 6; ties to the even code) and end at 6 scales.  Multiplying by a power of two is exact here: the inverse
// scale is a normal number for every s in use, and what falls below the binary32 range then rounds to code 0 as it would have.
// A block with Inf or NaN has s = 255 and codes 0.
//   k_mx4_step       d = grad - g, C(d), g += C(d), ||d - C(d)||^2 (Eq. 4, Eq. 6 with this compressor)
//   k_mx4_stats      the layers' errors and the workers' records from the CTAs' sums
//   k_mx4_apply      u^_m += C_m for every sender, and the model step (Algorithm 1, server lines)
//   k_mx4_read       a message as dense values
//   k_mx4_quantize_rows / _cols, k_mx4_dequantize_rows / _cols   operands (kimad_mx4_product.cuh multiplies them)
// All of them stream HBM once.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp4.h>

#include "kimad_kernels.cuh"

namespace kimad {

constexpr uint32_t kMxBlock = 32;      // values that share a scale
constexpr uint32_t kMxAbsent = 255;    // scale byte of a block with Inf or NaN
constexpr uint32_t kMxPieces = 16;     // CTAs of a chunk at most (k_mx4_step)
constexpr uint32_t kMxGroup = 8;       // blocks that a warp has in hand: one value of each per lane

struct MxPartial { // of a CTA of k_mx4_step
    double err;
    uint32_t absent, _pad;
};

template <typename T> __device__ __forceinline__ float mx_load(const T* p);
template <> __device__ __forceinline__ float mx_load<float>(const float* p) { return __ldcs(p); }
template <> __device__ __forceinline__ float mx_load<__nv_bfloat16>(const __nv_bfloat16* p) { return __bfloat162float(__ldcs(p)); }
template <> __device__ __forceinline__ float mx_load<__half>(const __half* p) { return __half2float(__ldcs(p)); }
__device__ __forceinline__ void mx_store(float* p, float v) { __stcs(p, v); }
__device__ __forceinline__ void mx_store(__nv_bfloat16* p, float v) { __stcs(p, __float2bfloat16_rn(v)); }

// Scale byte of a block whose largest magnitude has these bits, its inverse (0 where the block is absent) and its value.
__device__ __forceinline__ uint32_t mx_byte(uint32_t top) {
    const uint32_t e = top >> 23;
    return e >= 255u ? kMxAbsent : (e > 2u ? e - 2u : 0u);
}
__device__ __forceinline__ float mx_inverse(uint32_t byte) { return byte == kMxAbsent ? 0.f : __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ float mx_scale(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 1u << 22); } // byte 0: 2^-127, subnormal

// Two scaled values as two codes, the first one in the low half.
__device__ __forceinline__ uint32_t mx_pair(float lo, float hi) {
    return (uint32_t)__nv_cvt_float2_to_fp4x2(make_float2(lo, hi), __NV_E2M1, cudaRoundNearest);
}
__device__ __forceinline__ float2 mx_values(uint32_t pair) {
    const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)(pair & 0xffu), __NV_E2M1);
    return __half22float2(__half2(h));
}

// Eight lanes with eight codes each (nibble i of lane n) exchange them: lane i then has nibble n from lane n.  Three rounds of a butterfly, each
// swapping the halves whose index bits differ.
__device__ __forceinline__ uint32_t mx_transpose(uint32_t w, uint32_t lane) {
    auto round = [&](uint32_t s, uint32_t low) {
        const uint32_t p = __shfl_xor_sync(0xffffffffu, w, s);
        w = lane & s ? (w & ~low) | ((p & ~low) >> (4u * s)) : (w & low) | ((p & low) << (4u * s));
    };
    round(4, 0x0000ffffu);
    round(2, 0x00ff00ffu);
    round(1, 0x0f0f0f0fu);
    return w;
}

// The blocks of a chunk: those that start inside it.  They may reach into the layer's next chunk.
struct MxSpan {
    uint64_t base;   // flat index of the first block's first element
    uint64_t first;  // the first block's place in the worker's message
    uint32_t blocks, left; // elements from base on that are the layer's
    __device__ __forceinline__ MxSpan(const Chunk& ch, const LayerDesc& ld) {
        const uint64_t b0 = (ch.begin - ld.begin + kMxBlock - 1) / kMxBlock, b1 = (ch.end - ld.begin + kMxBlock - 1) / kMxBlock;
        base = ld.begin + b0 * kMxBlock;
        first = ch.block;
        blocks = (uint32_t)(b1 - b0);
        left = blocks ? (uint32_t)min(ld.n - b0 * kMxBlock, (uint64_t)blocks * kMxBlock) : 0u;
    }
};

// One CTA per chunk, or per piece of one (1 << log_pieces of them) where the chunks are few.  A warp takes eight blocks at a time, lane t the
// element t of each: every load and store is one line of consecutive elements whatever the alignment, a block's largest magnitude is one
// reduction over the warp, and eight lanes exchange nibbles so that each writes a word of codes.  Bound by HBM: 12.53 bytes per element with f32
// gradients, 10.53 with 16-bit ones.  The difference d - C(d) is exact in binary32 (C(d) is zero or a multiple of half a scale beside
// d), its squares are added in binary64: per thread, per CTA, per layer, always in the same order.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_mx4_step(const T* __restrict__ grads, float* __restrict__ state, uint64_t stride, const Chunk* __restrict__ chunks,
           const LayerDesc* __restrict__ layers, uint32_t log_pieces, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
           uint64_t code_bytes, uint64_t scale_bytes, MxPartial* __restrict__ partial) {
    pdl_wait();
    __shared__ double s_err[kThreads / 32];
    __shared__ uint32_t s_absent[kThreads / 32];
    const uint32_t w = blockIdx.y, f = blockIdx.x >> log_pieces, pieces = 1u << log_pieces, piece = blockIdx.x & (pieces - 1u);
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Chunk ch = chunks[f];
    const MxSpan sp(ch, layers[ch.layer]);
    const T* g = grads + (size_t)w * stride + sp.base;
    float* st = state + (size_t)w * stride + sp.base;
    uint32_t* cw = reinterpret_cast<uint32_t*>(codes + (size_t)w * code_bytes) + sp.first * 4;
    uint8_t* sc = scales + (size_t)w * scale_bytes + sp.first;
    double err = 0.0;
    uint32_t absent = 0;
    for (uint32_t b = (piece * (kThreads / 32) + warp) * kMxGroup; b < sp.blocks; b += pieces * (kThreads / 32) * kMxGroup) {
        const uint32_t e0 = b * kMxBlock + lane;
        float d[kMxGroup], s[kMxGroup];
#pragma unroll
        for (uint32_t i = 0; i < kMxGroup; ++i) {
            const uint32_t e = e0 + i * kMxBlock;
            const bool in = e < sp.left;
            s[i] = in ? __ldcs(st + e) : 0.f;
            d[i] = in ? mx_load(g + e) : 0.f;
        }
        uint32_t word = 0, mine = 0;
#pragma unroll
        for (uint32_t i = 0; i < kMxGroup; i += 2) {
            float r[2], x[2];
            uint32_t byte[2];
#pragma unroll
            for (uint32_t u = 0; u < 2; ++u) {
                d[i + u] = __fsub_rn(d[i + u], s[i + u]);
                byte[u] = mx_byte(__reduce_max_sync(0xffffffffu, key_of(d[i + u])));
                r[u] = byte[u] == kMxAbsent ? 0.f : __fmul_rn(d[i + u], mx_inverse(byte[u]));
                x[u] = mx_scale(byte[u]);
                if (lane == i + u) mine = byte[u];
            }
            const uint32_t pair = mx_pair(r[0], r[1]);
            word |= pair << (4u * i);
            const float2 q = mx_values(pair);
#pragma unroll
            for (uint32_t u = 0; u < 2; ++u) {
                const uint32_t e = e0 + (i + u) * kMxBlock;
                const float v = __fmul_rn(u ? q.y : q.x, x[u]);
                if (byte[u] == kMxAbsent) { absent += lane == 0; continue; }
                if (e < sp.left) __stcs(st + e, __fadd_rn(s[i + u], v));
                const double off = (double)__fsub_rn(d[i + u], v);
                err = fma(off, off, err);
            }
        }
        word = mx_transpose(word, lane);
        const uint32_t own = b + (lane & 7u);
        if (own < sp.blocks && KIMAD_CHECK((sp.first + own) * 16 + 16 <= code_bytes, 8)) cw[(size_t)own * 4 + (lane >> 3)] = word;
        if (lane < kMxGroup && b + lane < sp.blocks && KIMAD_CHECK(sp.first + b + lane < scale_bytes, 8)) sc[b + lane] = (uint8_t)mine;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) err += __shfl_xor_sync(0xffffffffu, err, o);
    if (lane == 0) { s_err[warp] = err; s_absent[warp] = absent; }
    __syncthreads();
    if (threadIdx.x == 0) {
        MxPartial p{0.0, 0, 0};
        for (int i = 0; i < kThreads / 32; ++i) { p.err += s_err[i]; p.absent += s_absent[i]; }
        partial[((size_t)w * (gridDim.x >> log_pieces) + f) * kMxPieces + piece] = p;
    }
}

// One CTA per worker.  A thread adds up the sums of a layer of few, a warp those of one with many; the order depends on the layers only.  A layer
// with an absent block has an infinite error, as its difference has.
constexpr int kMxStatsThreads = 1024;
__global__ void __launch_bounds__(kMxStatsThreads)
k_mx4_stats(const MxPartial* __restrict__ partial, const LayerDesc* __restrict__ layers, uint32_t L, uint32_t n_chunks, uint32_t log_pieces,
            uint64_t n, uint64_t message_bytes, uint32_t check_finite, float* __restrict__ err, kimad_stats* __restrict__ stats) {
    pdl_wait();
    __shared__ double s_err[kMxStatsThreads / 32];
    __shared__ uint32_t s_absent[kMxStatsThreads / 32];
    constexpr uint32_t kFew = 8; // sums that a thread adds up by itself
    const uint32_t w = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, pieces = 1u << log_pieces;
    const MxPartial* mine = partial + (size_t)w * n_chunks * kMxPieces;
    double total = 0.0;
    uint32_t absent = 0;
    auto done = [&](uint32_t l, double sum, uint32_t gone) {
        if (gone) sum = (double)__int_as_float(0x7f800000);
        err[(size_t)w * L + l] = (float)sum;
        total += sum;
        absent += gone;
    };
    for (uint32_t l = threadIdx.x; l < L; l += kMxStatsThreads) {
        const LayerDesc ld = layers[l];
        if (ld.n_chunks * pieces > kFew) continue;
        double sum = 0.0;
        uint32_t gone = 0;
        for (uint32_t i = 0; i < ld.n_chunks * pieces; ++i) {
            const MxPartial p = mine[(size_t)(ld.first_chunk + (i >> log_pieces)) * kMxPieces + (i & (pieces - 1u))];
            sum += p.err;
            gone += p.absent;
        }
        done(l, sum, gone);
    }
    for (uint32_t l = warp; l < L; l += kMxStatsThreads / 32) {
        const LayerDesc ld = layers[l];
        if (ld.n_chunks * pieces <= kFew) continue;
        double sum = 0.0;
        uint32_t gone = 0;
#pragma unroll 4
        for (uint32_t i = lane; i < ld.n_chunks * pieces; i += 32) {
            const MxPartial p = mine[(size_t)(ld.first_chunk + (i >> log_pieces)) * kMxPieces + (i & (pieces - 1u))];
            sum += p.err;
            gone += p.absent;
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, o);
            gone += __shfl_xor_sync(0xffffffffu, gone, o);
        }
        if (lane == 0) done(l, sum, gone);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        total += __shfl_xor_sync(0xffffffffu, total, o);
        absent += __shfl_xor_sync(0xffffffffu, absent, o);
    }
    if (lane == 0) { s_err[warp] = total; s_absent[warp] = absent; }
    __syncthreads();
    if (threadIdx.x == 0) {
        total = 0.0;
        absent = 0;
        for (int i = 0; i < kMxStatsThreads / 32; ++i) { total += s_err[i]; absent += s_absent[i]; }
        kimad_stats s{};
        s.used_bytes = message_bytes;
        s.n_selected = n;
        s.total_err = (float)total;
        s.status = absent && check_finite ? KIMAD_ERR_NONFINITE : KIMAD_OK;
        stats[w] = s;
    }
}

// Eight blocks of a message in a warp's hands: the values of element `lane` of each, and which blocks are absent (bit i).
__device__ __forceinline__ void mx_fetch(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, uint64_t first, uint32_t b, uint32_t blocks,
                                             uint32_t lane, uint32_t& word, uint32_t& byte) {
    const uint32_t own = b + (lane & 7u);
    word = own < blocks ? __ldcs(reinterpret_cast<const uint32_t*>(codes) + (first + own) * 4 + (lane >> 3)) : 0u;
    byte = own < blocks ? (uint32_t)__ldcs(scales + first + own) : kMxAbsent;
}
__device__ __forceinline__ uint32_t mx_decode(uint32_t word, uint32_t byte, uint32_t lane, float (&v)[kMxGroup]) {
    word = mx_transpose(word, lane);
    uint32_t gone = 0;
#pragma unroll
    for (uint32_t i = 0; i < kMxGroup; i += 2) {
        const float2 q = mx_values(word >> (4u * i));
        const uint32_t b0 = __shfl_sync(0xffffffffu, byte, i), b1 = __shfl_sync(0xffffffffu, byte, i + 1);
        v[i] = b0 == kMxAbsent ? 0.f : __fmul_rn(q.x, mx_scale(b0));
        v[i + 1] = b1 == kMxAbsent ? 0.f : __fmul_rn(q.y, mx_scale(b1));
        gone |= (b0 == kMxAbsent ? 1u << i : 0u) | (b1 == kMxAbsent ? 2u << i : 0u);
    }
    return gone;
}

struct MxWeights { float w[KIMAD_MAX_AGG_WORKERS]; };

// Same cut of the work as k_mx4_step.  Without the model a CTA has one sender (blockIdx.y); with it, all of them: an estimator's entry is then read
// and written once, and the model step (the order of k_aggregate's operations) costs the model's own 8 bytes instead of another
// pass over all estimators.  Two senders are in flight at a time.  An absent block leaves its estimator as it is.
template <bool MODEL>
__global__ void __launch_bounds__(kThreads)
k_mx4_apply(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, uint64_t code_bytes, uint64_t scale_bytes,
            const Chunk* __restrict__ chunks, const LayerDesc* __restrict__ layers, uint32_t log_pieces, float* __restrict__ est, uint64_t stride,
            uint32_t W, float* __restrict__ x, MxWeights wt, float gamma) {
    pdl_wait();
    constexpr uint32_t U = MODEL ? 2 : 1;
    const uint32_t f = blockIdx.x >> log_pieces, pieces = 1u << log_pieces, piece = blockIdx.x & (pieces - 1u);
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Chunk ch = chunks[f];
    const MxSpan sp(ch, layers[ch.layer]);
    const uint32_t m_first = MODEL ? 0u : blockIdx.y, m_end = MODEL ? W : blockIdx.y + 1u;
    for (uint32_t b = (piece * (kThreads / 32) + warp) * kMxGroup; b < sp.blocks; b += pieces * (kThreads / 32) * kMxGroup) {
        const uint32_t e0 = b * kMxBlock + lane;
        float acc[kMxGroup], xv[kMxGroup];
#pragma unroll
        for (uint32_t i = 0; i < kMxGroup; ++i) {
            acc[i] = 0.f;
            const uint32_t e = e0 + i * kMxBlock;
            xv[i] = MODEL && e < sp.left ? __ldcs(x + sp.base + e) : 0.f;
        }
        for (uint32_t m0 = m_first; m0 < m_end; m0 += U) {
            uint32_t word[U], byte[U];
            float s[U][kMxGroup];
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) {
                const uint32_t m = min(m0 + u, m_end - 1u);
                mx_fetch(codes + (size_t)m * code_bytes, scales + (size_t)m * scale_bytes, sp.first, b, sp.blocks, lane, word[u], byte[u]);
                const float* at = est + (size_t)m * stride + sp.base;
#pragma unroll
                for (uint32_t i = 0; i < kMxGroup; ++i) {
                    const uint32_t e = e0 + i * kMxBlock;
                    s[u][i] = e < sp.left && m0 + u < m_end ? __ldcs(at + e) : 0.f;
                }
            }
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) {
                if (m0 + u >= m_end) break;
                float v[kMxGroup];
                const uint32_t gone = mx_decode(word[u], byte[u], lane, v);
                float* at = est + (size_t)(m0 + u) * stride + sp.base;
                const float wm = MODEL ? wt.w[m0 + u] : 0.f;
#pragma unroll
                for (uint32_t i = 0; i < kMxGroup; ++i) {
                    const uint32_t e = e0 + i * kMxBlock;
                    if (!(gone >> i & 1u)) {
                        s[u][i] = __fadd_rn(s[u][i], v[i]);
                        if (e < sp.left) __stcs(at + e, s[u][i]);
                    }
                    if (MODEL) acc[i] = __fadd_rn(acc[i], __fmul_rn(wm, s[u][i]));
                }
            }
        }
        if (MODEL) {
#pragma unroll
            for (uint32_t i = 0; i < kMxGroup; ++i) {
                const uint32_t e = e0 + i * kMxBlock;
                if (e < sp.left) __stcs(x + sp.base + e, __fsub_rn(xv[i], __fmul_rn(gamma, acc[i])));
            }
        }
    }
}

// C(d) as dense values (0 where a block is absent).  bfloat16 holds every one of them exactly: two significant bits and bfloat16's exponents.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_mx4_read(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, uint64_t code_bytes, uint64_t scale_bytes,
           const Chunk* __restrict__ chunks, const LayerDesc* __restrict__ layers, uint32_t log_pieces, T* __restrict__ out, uint64_t stride) {
    pdl_wait();
    const uint32_t w = blockIdx.y, f = blockIdx.x >> log_pieces, pieces = 1u << log_pieces, piece = blockIdx.x & (pieces - 1u);
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Chunk ch = chunks[f];
    const MxSpan sp(ch, layers[ch.layer]);
    T* o = out + (size_t)w * stride + sp.base;
    for (uint32_t b = (piece * (kThreads / 32) + warp) * kMxGroup; b < sp.blocks; b += pieces * (kThreads / 32) * kMxGroup) {
        const uint32_t e0 = b * kMxBlock + lane;
        uint32_t word, byte;
        float v[kMxGroup];
        mx_fetch(codes + (size_t)w * code_bytes, scales + (size_t)w * scale_bytes, sp.first, b, sp.blocks, lane, word, byte);
        mx_decode(word, byte, lane, v);
#pragma unroll
        for (uint32_t i = 0; i < kMxGroup; ++i) {
            const uint32_t e = e0 + i * kMxBlock;
            if (e < sp.left) mx_store(o + e, v[i]);
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
    // the four scales of a line in a tile of blocks, as a word
    KIMAD_HD uint64_t scale_word(uint32_t line, uint32_t tile) const {
        return ((uint64_t)(line / kMxTile) * block_tiles + tile) * 128 + (line % 32) * 4 + line % kMxTile / 32;
    }
};

// Blocks along the contiguous axis: a warp takes eight of a line, as in k_mx4_step.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_mx4_quantize_rows(const T* __restrict__ x, uint64_t ld, uint64_t batch_stride, uint64_t batch, MxOperand op, uint8_t* __restrict__ codes,
                    uint8_t* __restrict__ scales) {
    pdl_wait();
    const uint32_t lane = threadIdx.x & 31;
    const uint32_t segs = (op.blocks + kMxGroup - 1) / kMxGroup, lines = op.line_tiles * kMxTile;
    const uint64_t all = batch * lines * segs, step = (uint64_t)gridDim.x * (kThreads / 32);
    for (uint64_t at = (uint64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); at < all; at += step) {
        const uint32_t seg = (uint32_t)(at % segs), line = (uint32_t)(at / segs % lines);
        const uint64_t n = at / segs / lines;
        const uint32_t b = seg * kMxGroup;
        uint32_t word = 0, lo = 0, hi = 0; // codes, scales of blocks 0-3 and 4-7
        if (line < op.lines) {
            const T* row = x + n * batch_stride + (uint64_t)line * ld;
            float v[kMxGroup];
#pragma unroll
            for (uint32_t i = 0; i < kMxGroup; ++i) {
                const uint64_t e = (uint64_t)(b + i) * kMxBlock + lane;
                v[i] = e < op.length ? mx_load(row + e) : 0.f;
            }
#pragma unroll
            for (uint32_t i = 0; i < kMxGroup; i += 2) {
                float r[2];
#pragma unroll
                for (uint32_t u = 0; u < 2; ++u) {
                    const uint32_t byte = mx_byte(__reduce_max_sync(0xffffffffu, key_of(v[i + u])));
                    r[u] = byte == kMxAbsent ? 0.f : __fmul_rn(v[i + u], mx_inverse(byte));
                    if (i < 4) lo |= byte << (8 * (i + u));
                    else hi |= byte << (8 * (i + u - 4));
                }
                word |= mx_pair(r[0], r[1]) << (4u * i);
            }
            word = mx_transpose(word, lane);
            const uint32_t own = b + (lane & 7u);
            if (own < op.blocks)
                reinterpret_cast<uint32_t*>(codes)[((n * op.lines + line) * op.blocks + own) * 4 + (lane >> 3)] = word;
        }
        if (lane < 2 && seg * 2 + lane < op.block_tiles)
            reinterpret_cast<uint32_t*>(scales)[n * (op.scale_bytes() / 4) + op.scale_word(line, seg * 2 + lane)] = lane ? hi : lo;
    }
}

// Blocks along the other axis, which transposes: a CTA takes 128 lines (columns of x) by 128 values (rows), a lane one block of a column.  Rows are
// read in whole lines and need no exchange between lanes; codes go through shared memory so that 64 bytes of a line are written together.
constexpr int kMxColThreads = 512;
template <typename T>
__global__ void __launch_bounds__(kMxColThreads)
k_mx4_quantize_cols(const T* __restrict__ x, uint64_t ld, uint64_t batch_stride, MxOperand op, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    pdl_wait();
    __shared__ uint4 s_codes[kMxTile][4];
    __shared__ uint8_t s_scales[512];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t lt = blockIdx.x % op.line_tiles, bt = blockIdx.x / op.line_tiles % op.block_tiles;
    const uint64_t n = blockIdx.x / op.line_tiles / op.block_tiles;
    const uint32_t in_line = (warp & 3u) * 32 + lane, line = lt * kMxTile + in_line, q = warp >> 2, block = bt * 4 + q;
    float v[kMxBlock];
    uint32_t top = 0;
    const T* from = x + n * batch_stride + line;
#pragma unroll
    for (uint32_t i = 0; i < kMxBlock; ++i) {
        const uint64_t row = (uint64_t)block * kMxBlock + i;
        v[i] = line < op.lines && row < op.length ? mx_load(from + row * ld) : 0.f;
    }
#pragma unroll
    for (uint32_t i = 0; i < kMxBlock; ++i) top = max(top, key_of(v[i]));
    const uint32_t byte = mx_byte(top);
    const float inv = mx_inverse(byte);
    uint32_t word[4] = {};
    if (byte != kMxAbsent) {
#pragma unroll
        for (uint32_t i = 0; i < kMxBlock; i += 2) word[i / 8] |= mx_pair(__fmul_rn(v[i], inv), __fmul_rn(v[i + 1], inv)) << (4u * (i % 8));
    }
    s_codes[in_line][q] = make_uint4(word[0], word[1], word[2], word[3]);
    s_scales[in_line % 32 * 16 + in_line / 32 * 4 + q] = (uint8_t)byte;
    __syncthreads();
    const uint32_t out_line = threadIdx.x / 4, out_block = threadIdx.x % 4;
    if (lt * kMxTile + out_line < op.lines && bt * 4 + out_block < op.blocks)
        reinterpret_cast<uint4*>(codes)[(n * op.lines + lt * kMxTile + out_line) * op.blocks + bt * 4 + out_block] = s_codes[out_line][out_block];
    if (threadIdx.x < 128)
        reinterpret_cast<uint32_t*>(scales)[((n * op.line_tiles + lt) * op.block_tiles + bt) * 128 + threadIdx.x] = reinterpret_cast<uint32_t*>(s_scales)[threadIdx.x];
}

// Back to values, both ways round.  A block that could not be quantised reads as NaN.
__device__ __forceinline__ float mx_operand_scale(uint32_t byte) { return byte == kMxAbsent ? __int_as_float(0x7fffffff) : mx_scale(byte); }

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_mx4_dequantize_rows(T* __restrict__ x, uint64_t ld, uint64_t batch_stride, uint64_t batch, MxOperand op, const uint8_t* __restrict__ codes,
                      const uint8_t* __restrict__ scales) {
    pdl_wait();
    const uint32_t lane = threadIdx.x & 31, segs = (op.blocks + kMxGroup - 1) / kMxGroup;
    const uint64_t all = batch * op.lines * segs, step = (uint64_t)gridDim.x * (kThreads / 32);
    for (uint64_t at = (uint64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); at < all; at += step) {
        const uint32_t seg = (uint32_t)(at % segs), line = (uint32_t)(at / segs % op.lines);
        const uint64_t n = at / segs / op.lines;
        const uint32_t b = seg * kMxGroup, own = b + (lane & 7u);
        uint32_t word = own < op.blocks ? __ldcs(reinterpret_cast<const uint32_t*>(codes) + ((n * op.lines + line) * op.blocks + own) * 4 + (lane >> 3)) : 0u;
        const uint32_t four = lane < 2 && seg * 2 + lane < op.block_tiles
                                  ? __ldcs(reinterpret_cast<const uint32_t*>(scales) + n * (op.scale_bytes() / 4) + op.scale_word(line, seg * 2 + lane)) : 0u;
        const uint32_t lo = __shfl_sync(0xffffffffu, four, 0), hi = __shfl_sync(0xffffffffu, four, 1);
        word = mx_transpose(word, lane);
        T* row = x + n * batch_stride + (uint64_t)line * ld;
#pragma unroll
        for (uint32_t i = 0; i < kMxGroup; i += 2) {
            const float2 q = mx_values(word >> (4u * i));
#pragma unroll
            for (uint32_t u = 0; u < 2; ++u) {
                const uint64_t e = (uint64_t)(b + i + u) * kMxBlock + lane;
                const uint32_t byte = ((i < 4 ? lo : hi) >> (8 * ((i + u) % 4))) & 255u;
                if (e < op.length) mx_store(row + e, __fmul_rn(u ? q.y : q.x, mx_operand_scale(byte)));
            }
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kMxColThreads)
k_mx4_dequantize_cols(T* __restrict__ x, uint64_t ld, uint64_t batch_stride, MxOperand op, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales) {
    pdl_wait();
    __shared__ uint4 s_codes[kMxTile][4];
    __shared__ uint32_t s_scales[128];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t lt = blockIdx.x % op.line_tiles, bt = blockIdx.x / op.line_tiles % op.block_tiles;
    const uint64_t n = blockIdx.x / op.line_tiles / op.block_tiles;
    const uint32_t in = threadIdx.x / 4, in_block = threadIdx.x % 4;
    if (lt * kMxTile + in < op.lines && bt * 4 + in_block < op.blocks)
        s_codes[in][in_block] = __ldcs(reinterpret_cast<const uint4*>(codes) + (n * op.lines + lt * kMxTile + in) * op.blocks + bt * 4 + in_block);
    if (threadIdx.x < 128) s_scales[threadIdx.x] = __ldcs(reinterpret_cast<const uint32_t*>(scales) + ((n * op.line_tiles + lt) * op.block_tiles + bt) * 128 + threadIdx.x);
    __syncthreads();
    const uint32_t in_line = (warp & 3u) * 32 + lane, line = lt * kMxTile + in_line, q = warp >> 2, block = bt * 4 + q;
    if (line >= op.lines || block >= op.blocks) return;
    const uint4 c = s_codes[in_line][q];
    const uint32_t word[4] = {c.x, c.y, c.z, c.w};
    const float scale = mx_operand_scale((s_scales[in_line % 32 * 4 + in_line / 32] >> (8 * q)) & 255u);
    T* to = x + n * batch_stride + line;
#pragma unroll
    for (uint32_t i = 0; i < kMxBlock; i += 2) {
        const float2 v = mx_values(word[i / 8] >> (4u * (i % 8)));
        const uint64_t row = (uint64_t)block * kMxBlock + i;
        if (row < op.length) mx_store(to + row * ld, __fmul_rn(v.x, scale));
        if (row + 1 < op.length) mx_store(to + (row + 1) * ld, __fmul_rn(v.y, scale));
    }
}

} // namespace kimad
