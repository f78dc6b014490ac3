// Layout of the paged 4-bit key/value cache and the device helpers that its kernels share (see include/asymgemm.h,
// "4-bit key/value cache in pages", for the layout as users see it).
//
// Codes lie in the order in which a warp's lanes hold the operands of the 16 x 8 x 16 MMA of the decode attention: lane
// 4 g + t finds its share of a run of 16 tokens as two runs of D / 8 contiguous bytes (h = 0, 1), so that a shared-memory
// load of the fragments is one conflict-free vector load a lane, and a whole page of a head is one contiguous copy.
#pragma once
#include <cuda_bf16.h>
#include <string.h>

#include "internal.h"
#include "ptx.cuh"

namespace ag {

constexpr int KV4_PAGE = AG_KV4_PAGE;      // tokens per page
constexpr int KV4_GROUP = 32;              // elements that share a scale and a base

__host__ __device__ constexpr int kv4_head_bytes(int D) { return 80 * D; }
// byte offset, inside a head's block, of the codes of token `tok` for lane part (g of the operand, t) and of its scales
template <int D>
__device__ __forceinline__ int kv4_k_word(int tok, int grp, int t) {         // elements 32 grp + 8 t + 0 .. 7 of K: one word
    return tok * (D / 2) + t * (D / 8) + 4 * grp;                            // = (tok / 16) 8 D + (tok / 8 % 2) 4 D + (4 (tok % 8) + t) D / 8 + 4 grp
}
template <int D>
__device__ __forceinline__ int kv4_v_word(int tok, int hi, int g) {          // elements 16 i + 8 hi + g of V, all i: D / 32 bytes
    return 32 * D + (tok >> 3) * 4 * D + (4 * g + ((tok >> 1) & 3)) * (D / 8) + (tok & 1) * (D / 16) + hi * (D / 32);
}
template <int D>
__device__ __forceinline__ int kv4_scale_word(int which, int tok, int grp) { // (scale, base) as a pair of bf16
    return 64 * D + which * 8 * D + (tok * (D / 32) + grp) * 4;
}

// A 4-bit matrix, one row a lane (index i = lane position among the N lanes that exchange with lane ^ (STEP << s)), is
// transposed in blocks of N x N by halving: afterwards the lane's block holds column i.  Its own inverse.
template <int N, int STEP>
__device__ __forceinline__ uint32_t kv4_transpose(uint32_t w, int i) {
    if (N == 8) {
        const uint32_t o = __shfl_xor_sync(0xffffffffu, w, 4 * STEP);
        w = (i & 4) ? (w & 0xffff0000u) | (o >> 16) : (w & 0x0000ffffu) | (o << 16);
    }
    {
        const uint32_t o = __shfl_xor_sync(0xffffffffu, w, 2 * STEP);
        w = (i & 2) ? (w & 0xff00ff00u) | ((o >> 8) & 0x00ff00ffu) : (w & 0x00ff00ffu) | ((o << 8) & 0xff00ff00u);
    }
    {
        const uint32_t o = __shfl_xor_sync(0xffffffffu, w, STEP);
        w = (i & 1) ? (w & 0xf0f0f0f0u) | ((o >> 4) & 0x0f0f0f0fu) : (w & 0x0f0f0f0fu) | ((o << 4) & 0xf0f0f0f0u);
    }
    return w;
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Quantisation of a group x_0 .. x_31: lo = min, s = bf16((max - lo) / 15), code = rint((x - lo) / s) in 0 .. 15, and an element
// stands for s code + lo.  lo is an element, so it is a bf16 already; s is rounded to bf16 first and the codes are taken for the
// rounded one, so that the rounding costs at most 2^-9 of a step.  All in 32 bits with IEEE rounding: the codes do not depend on the kernel.
// A group with a value that is not finite, or whose range is not, stands for NaN throughout.
__device__ __forceinline__ uint32_t min_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// D / 16 lanes hold a row (which = 0: of K, 1: of V), lane l its elements 16 l .. 16 l + 15; all lanes of the warp take part.  The lane's two words of
// codes, V's transposed already, and the (scale, base) pair of the lane's group.
template <int D>
__device__ __forceinline__ uint32_t kv4_quantise(const uint32_t (&in)[8], int which, int l, uint32_t (&w)[2]) {
    // extremes of the group, in pairs; NaN wins, and an infinity makes the range infinite or NaN
    uint32_t lo2 = in[0], hi2 = in[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        lo2 = min_bf16x2(lo2, in[i]);
        hi2 = max_bf16x2(hi2, in[i]);
    }
    lo2 = min_bf16x2(lo2, __shfl_xor_sync(0xffffffffu, lo2, 1));
    hi2 = max_bf16x2(hi2, __shfl_xor_sync(0xffffffffu, hi2, 1));
    const float lo = bf16_lo(min_bf16x2(lo2, lo2 >> 16)), hi = bf16_lo(max_bf16x2(hi2, hi2 >> 16));
    const __nv_bfloat16 sb = __float2bfloat16_rn(__fdiv_rn(__fsub_rn(hi, lo), 15.f));
    const float s = __bfloat162float(sb);
    const bool fine = s <= 3.4e38f;                             // false for NaN and infinity
    // rint((x - lo) / s): the quotient from the correctly rounded reciprocal and one step on the exact remainder, which is the correctly
    // rounded quotient (Markstein) while nothing over- or underflows; four codes are gathered as one number in base 16.
    w[0] = w[1] = 0;
    if (s >= 0x1p-90f && s <= 0x1p100f) {
        constexpr float M = 12582912.f;                         // 1.5 * 2^23: adding it rounds to an integer, halves to even
        const float inv = __frcp_rn(s);
        float number[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 15; i >= 0; --i) {
            const float d = __fsub_rn(i & 1 ? bf16_hi(in[i >> 1]) : bf16_lo(in[i >> 1]), lo);
            const float q1 = __fmul_rn(d, inv), q = __fmaf_rn(__fmaf_rn(-q1, s, d), inv, q1);
            number[i >> 2] = __fmaf_rn(number[i >> 2], 16.f, __fsub_rn(__fadd_rn(q, M), M));
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
            w[k] = __byte_perm(__float_as_uint(number[2 * k] + 8388608.f), __float_as_uint(number[2 * k + 1] + 8388608.f), 0x5410);
    } else if (fine && s > 0.f) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float d = __fsub_rn(i & 1 ? bf16_hi(in[i >> 1]) : bf16_lo(in[i >> 1]), lo);
            w[i >> 3] |= (uint32_t)min(15, __float2int_rn(__fdiv_rn(d, s))) << (4 * (i & 7));
        }
    }
    if (which) {                                                // lane l has elements 16 l + 8 j + g, word j: then word j holds elements 16 i + 8 j + l
        w[0] = kv4_transpose<D / 16, 1>(w[0], l);
        w[1] = kv4_transpose<D / 16, 1>(w[1], l);
    }
    const uint32_t pair = (uint32_t)__bfloat16_as_ushort(sb) | (__float_as_uint(lo) & 0xffff0000u);
    return fine ? pair : 0x7fc07fc0u;                               // a NaN for each
}
// Into a head's block, place r of its page.
template <int D>
__device__ __forceinline__ void kv4_put(uint8_t* block, int which, int r, int l, const uint32_t (&w)[2], uint32_t pair) {
    if (which == 0) {
        uint8_t* to = block + kv4_k_word<D>(r, l >> 1, 2 * (l & 1));
        *reinterpret_cast<uint32_t*>(to) = w[0];
        *reinterpret_cast<uint32_t*>(to + D / 8) = w[1];
    } else if (D == 128) {
        *reinterpret_cast<uint2*>(block + kv4_v_word<D>(r, 0, l)) = make_uint2(w[0], w[1]);
    } else {
        *reinterpret_cast<uint32_t*>(block + kv4_v_word<D>(r, 0, l)) = __byte_perm(w[0], w[1], 0x5410);
        *reinterpret_cast<uint32_t*>(block + kv4_v_word<D>(r, 0, 4 + l)) = __byte_perm(w[0], w[1], 0x7632);
    }
    if ((l & 1) == 0) *reinterpret_cast<uint32_t*>(block + kv4_scale_word<D>(which, r, l >> 1)) = pair;
}

// Waits until the launch before this one on the stream has completed (launches of this library with the programmatic
// attribute), and lets the next one come up.  A kernel that waits here takes no `__restrict__` pointers: what it reads may have been
// written while it was up already, and the qualifier would let the compiler read it in front of the wait or through a cache that is not coherent.
__device__ __forceinline__ void dep_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void dep_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

inline bool kv4_pool_ok(const ag_kv4_pool* p) {
    return p && p->pages && !((uintptr_t)p->pages & 15u) && p->n_pages >= 1 && p->n_pages < (1ll << 25) && p->H_kv >= 1 && p->H_kv <= 1024 &&
           (p->D == 64 || p->D == 128);
}
inline bool kv4_table_ok(const ag_kv4_table* t) {
    return t && t->page_of && t->len && t->refs && t->n_rows >= 1 && t->max_pages >= 1 && t->max_pages < (1 << 25) &&
           !(((uintptr_t)t->page_of | (uintptr_t)t->len | (uintptr_t)t->refs) & 3u);
}

// Launch that may come up while the launch before it on the stream finishes; the kernel itself waits for it (dep_wait) before it touches memory.
template <class... P, class... A>
inline cudaError_t launch_dependent(void (*kernel)(P...), unsigned grid, unsigned block, cudaStream_t stream, A... args) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

}  // namespace ag
