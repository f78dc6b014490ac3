// Layout of the paged 4-bit key/value cache and the device helpers that its kernels share (see include/asymgemm.h,
// "4-bit key/value cache in pages", for the layout as users see it).
//
// Codes lie in the order in which a warp's lanes hold the operands of the 16 x 8 x 16 MMA of the decode attention: lane
// 4 g + t finds its share of a run of 16 tokens as two runs of D / 8 contiguous bytes (h = 0, 1), so that a shared-memory
// load of the fragments is one conflict-free vector load a lane, and a whole page of a head is one contiguous copy.
#pragma once
#include <cuda_bf16.h>

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

}  // namespace ag
