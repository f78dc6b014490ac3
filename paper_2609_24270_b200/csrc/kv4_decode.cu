// Single-token attention over the paged 4-bit key/value cache (layout: kv4.cuh).
//
// Per request, KV head and page of 64 keys, with the code u and the pair (s, b) of every element (value s u + b), G query heads:
//     S[key][q]  = sum over groups of 32 d:  s (sum_d u q_d) + b (sum_d q_d)      m16n8k16 MMA: 16 keys x 8 heads x 16 d
//     P = 2^((S - max) log2 e / sqrt D)                                           running maximum and sum per warp
//     O[d][q]   += sum_key V[key][d] P[key][q]                                    m16n8k16 MMA: 16 d x 8 heads x 16 keys
// A code becomes a bf16 operand without arithmetic: 0x4300 | u is 128 + u.  For K the 128 leaves with the base, exactly (the
// group's sum of q is known in 32 bits): scores carry no rounding besides the 32-bit sums.  V is rounded to bf16 once (its scale varies
// along the contraction), P once; the sums are in 32 bits.
//
// Bound by memory: 1.25 D bytes per key and head.  A byte costs about ten times the arithmetic instructions of a bf16 cache's, so
// the operands are unpacked in registers, straight into the MMA's fragments - tcgen05.mma would want them in shared memory, one more
// write and read of the unpacked (four times larger) tile.  The cache stores the codes in fragment order, so a warp's share of a
// page is read with one conflict-free vector load a lane.  Every warp owns its pages (page w, w + 8, ... of the block's range) and one
// buffer each for K and V, refilled by 16-byte asynchronous copies as soon as it has been read: K of the next page comes in during the softmax and
// V's products, V during the next page's scores, with 16 warps an SM in different phases.  No block-wide step until the warps' results are
// put together.  Long requests are cut into splits (blocks); a second kernel joins them.
#include <string.h>

#include <algorithm>

#include "kv4.cuh"

namespace ag {

constexpr int DK_WARPS = 8;
constexpr int DK_MAXSPLIT = 128;

struct DecodeKv4Args {
    const uint16_t* Q;            // [B][H_q][D]
    uint16_t* O;                  // [B][H_q][D]
    const uint8_t* pages;
    const int32_t *page_of, *len, *row;
    float* part;                  // [units][splits][heads of a block][D] (splits > 1)
    float2* stats;                // [units][splits][heads of a block]: maximum (in units of log2), sum
    int n_pages, H_kv, G, n_rows, max_pages, n_split, h_blocks;
    float scale_log2e;
};

__device__ __forceinline__ float ex2_ftz(float v) {      // 2^v, relative error 2^-22; 2^-inf = 0
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t movm_trans(uint32_t v) {      // 8 x 8 matrix of 16-bit elements, transposed across the warp
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// nibbles `shift / 4` of both halves of w, each as the bf16 128 + u
__device__ __forceinline__ uint32_t codes128(uint32_t w, int shift) { return ((w >> shift) & 0x000f000fu) | 0x43004300u; }
__device__ __forceinline__ uint32_t dequant2(uint32_t c128, uint32_t s, uint32_t b) {
    const __nv_bfloat162 m128 = __halves2bfloat162(__ushort_as_bfloat16(0xC300), __ushort_as_bfloat16(0xC300));
    const __nv_bfloat162 u = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&c128), m128);
    const __nv_bfloat162 v = __hfma2(u, *reinterpret_cast<const __nv_bfloat162*>(&s), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// pages of a request that split `sp` of a unit covers; a split gets at least DK_WARPS pages
__device__ __forceinline__ int splits_in_use(int n_page, int n_split) { return max(1, min(n_split, (n_page + DK_WARPS - 1) / DK_WARPS)); }

template <int D, int NB>
constexpr int dk_smem_bytes() {
    return DK_WARPS * kv4_head_bytes(D) > DK_WARPS * 8 * NB * (D + 4) * 4 ? DK_WARPS * kv4_head_bytes(D) : DK_WARPS * 8 * NB * (D + 4) * 4;
}

template <int D, int NB>
__global__ void __launch_bounds__(DK_WARPS * 32, NB == 1 ? 2 : 1) k_attn_decode_kv4(const DecodeKv4Args x) {
    constexpr int NG = D / 32;                     // groups of a row
    constexpr int MT = D / 16;                     // tiles of 16 d
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ float2 warp_stat[DK_WARPS][8 * NB];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    dep_release();
    const int sp = blockIdx.x % x.n_split, unit = blockIdx.x / x.n_split;
    const int hb = unit % x.h_blocks, bh = unit / x.h_blocks;
    const int h = bh % x.H_kv, b = bh / x.H_kv;
    const int r = x.row ? x.row[b] : b;
    const bool known = r >= 0 && r < x.n_rows;
    const int len = known ? min(max(x.len[r], 0), x.max_pages * KV4_PAGE) : 0;
    const int n_page = (len + KV4_PAGE - 1) / KV4_PAGE;
    const int in_use = splits_in_use(n_page, x.n_split);
    if (sp >= in_use) return;                      // (the joining kernel knows)
    const int p_begin = (int)((long long)n_page * sp / in_use), p_end = (int)((long long)n_page * (sp + 1) / in_use);
    const int head0 = hb * 8 * NB;                 // first query head of the block, of the KV head's G
    const uint16_t* q_rows = x.Q + ((size_t)b * x.H_kv + h) * x.G * D;

    // ---- queries as B operands: lane (g, t) holds head g, elements 32 grp + 8 t + {0, 4}, {1, 5}, {2, 6}, {3, 7}
    uint32_t qf[NB][NG][4];
    float qsum[NB][NG][2];                         // sums of q over a group, heads 2 t and 2 t + 1
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int head = head0 + nb * 8 + g;
#pragma unroll
        for (int grp = 0; grp < NG; ++grp) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (head < x.G) v = *reinterpret_cast<const uint4*>(q_rows + (size_t)head * D + grp * 32 + t * 8);
            qf[nb][grp][0] = __byte_perm(v.x, v.z, 0x5410);
            qf[nb][grp][1] = __byte_perm(v.x, v.z, 0x7632);
            qf[nb][grp][2] = __byte_perm(v.y, v.w, 0x5410);
            qf[nb][grp][3] = __byte_perm(v.y, v.w, 0x7632);
            float s = ((bf16_lo(v.x) + bf16_hi(v.x)) + (bf16_lo(v.y) + bf16_hi(v.y))) + ((bf16_lo(v.z) + bf16_hi(v.z)) + (bf16_lo(v.w) + bf16_hi(v.w)));
            s += __shfl_xor_sync(0xffffffffu, s, 1);
            s += __shfl_xor_sync(0xffffffffu, s, 2);
            qsum[nb][grp][0] = __shfl_sync(0xffffffffu, s, 8 * t);
            qsum[nb][grp][1] = __shfl_sync(0xffffffffu, s, 8 * t + 4);
        }
    }

    uint8_t* kbuf = smem + warp * kv4_head_bytes(D);          // codes of K, then K's pairs
    uint8_t* vbuf = kbuf + 40 * D;
    const uint32_t kbuf_a = smem_u32(kbuf), vbuf_a = smem_u32(vbuf);
    const int32_t* ids = x.page_of + (size_t)(known ? r : 0) * x.max_pages;
    int id_batch = 0;
    // this warp's n-th page: its id and the keys of it that count
    auto page_at = [&](int n, int& id, int& nv) {
        const int p = p_begin + warp + n * DK_WARPS;
        if ((n & 31) == 0) {
            const int pl = p + lane * DK_WARPS;
            id_batch = pl < p_end ? ids[pl] : -1;
        }
        id = __shfl_sync(0xffffffffu, id_batch, n & 31);
        nv = p < p_end && id >= 0 && id < x.n_pages ? min(KV4_PAGE, len - p * KV4_PAGE) : 0;
    };
    // copies the runs of 16 tokens that hold keys: codes (8 D bytes a run) and pairs (2 D bytes a run)
    auto fetch = [&](int which, int id, int nv) {
        if (nv > 0) {
            const uint8_t* src = x.pages + ((size_t)id * x.H_kv + h) * kv4_head_bytes(D);
            const uint32_t dst = which ? vbuf_a : kbuf_a;
            const int runs = (nv + 15) >> 4;
            const uint8_t* codes = src + which * 32 * D + lane * 16;
            const uint8_t* pairs = src + 64 * D + which * 8 * D + lane * 16;
#pragma unroll
            for (int j = 0; j < 32 * D / 512; ++j)
                if (j * 512 < runs * 8 * D) cp_async16(dst + j * 512 + lane * 16, codes + j * 512);
#pragma unroll
            for (int j = 0; j < 8 * D / 512; ++j)
                if (j * 512 + lane * 16 < runs * 2 * D) cp_async16(dst + 32 * D + j * 512 + lane * 16, pairs + j * 512);
        }
        cp_async_commit();
    };

    float o[NB][MT][4];
    float m[NB][2], l[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) o[nb][i][c] = 0.f;
        m[nb][0] = m[nb][1] = -INFINITY;
        l[nb][0] = l[nb][1] = 0.f;
    }
    const int n_mine = p_end - p_begin > warp ? (p_end - p_begin - warp + DK_WARPS - 1) / DK_WARPS : 0;
    int id, nv, id_next = -1, nv_next = 0;
    if (n_mine > 0) {
        page_at(0, id, nv);
        fetch(0, id, nv);
        fetch(1, id, nv);
    }
    for (int n = 0; n < n_mine; ++n) {
        cp_async_wait<1>();                        // K of this page has landed
        __syncwarp();
        float s[NB][4][4];
#pragma unroll
        for (int run = 0; run < 4; ++run) {
            if (run * 16 < nv) {
                uint32_t w[2][NG], sb[2][NG];      // rows g and g + 8 of the run
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const uint8_t* at = kbuf + run * 8 * D + hh * 4 * D + lane * (D / 8);
                    const uint8_t* ps = kbuf + 32 * D + (run * 16 + hh * 8 + g) * (D / 8);
                    if (D == 128) {
                        *reinterpret_cast<uint4*>(&w[hh][0]) = *reinterpret_cast<const uint4*>(at);
                        *reinterpret_cast<uint4*>(&sb[hh][0]) = *reinterpret_cast<const uint4*>(ps);
                    } else {
                        *reinterpret_cast<uint2*>(&w[hh][0]) = *reinterpret_cast<const uint2*>(at);
                        *reinterpret_cast<uint2*>(&sb[hh][0]) = *reinterpret_cast<const uint2*>(ps);
                    }
                }
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int c = 0; c < 4; ++c) s[nb][run][c] = 0.f;
#pragma unroll
                for (int grp = 0; grp < NG; ++grp) {
                    const float s0 = bf16_lo(sb[0][grp]), s1 = bf16_lo(sb[1][grp]);
                    const float b0 = fmaf(-128.f, s0, bf16_hi(sb[0][grp])), b1 = fmaf(-128.f, s1, bf16_hi(sb[1][grp]));
                    uint32_t a[8];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        a[2 * k] = codes128(w[0][grp], 4 * k);
                        a[2 * k + 1] = codes128(w[1][grp], 4 * k);
                    }
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        float acc[4] = {0.f, 0.f, 0.f, 0.f};
                        mma_bf16(acc, a[0], a[1], a[2], a[3], qf[nb][grp][0], qf[nb][grp][1]);
                        mma_bf16(acc, a[4], a[5], a[6], a[7], qf[nb][grp][2], qf[nb][grp][3]);
                        s[nb][run][0] += fmaf(s0, acc[0], b0 * qsum[nb][grp][0]);
                        s[nb][run][1] += fmaf(s0, acc[1], b0 * qsum[nb][grp][1]);
                        s[nb][run][2] += fmaf(s1, acc[2], b1 * qsum[nb][grp][0]);
                        s[nb][run][3] += fmaf(s1, acc[3], b1 * qsum[nb][grp][1]);
                    }
                }
            }
        }
        __syncwarp();                              // every lane has read K
        if (n + 1 < n_mine) page_at(n + 1, id_next, nv_next);
        else nv_next = 0;
        fetch(0, id_next, nv_next);
        if (nv > 0) {
            // ---- softmax: keys past the end count as -inf
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float top[2] = {m[nb][0], m[nb][1]};
#pragma unroll
                for (int run = 0; run < 4; ++run)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const float v = run * 16 + g + (c >> 1) * 8 < nv ? s[nb][run][c] * x.scale_log2e : -INFINITY;
                        s[nb][run][c] = v;
                        top[c & 1] = fmaxf(top[c & 1], v);
                    }
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int w = 4; w < 32; w <<= 1) top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], w));
                float f[2], ref[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    ref[e] = top[e] == -INFINITY ? 0.f : top[e];
                    f[e] = ex2_ftz(m[nb][e] - ref[e]);
                }
                if (__any_sync(0xffffffffu, top[0] != m[nb][0] || top[1] != m[nb][1])) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        l[nb][e] *= f[e];
                        m[nb][e] = top[e];
                    }
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int c = 0; c < 4; ++c) o[nb][i][c] *= f[c & 1];
                }
#pragma unroll
                for (int run = 0; run < 4; ++run)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        s[nb][run][c] = ex2_ftz(s[nb][run][c] - ref[c & 1]);
                        l[nb][c & 1] += s[nb][run][c];
                    }
            }
        }
        cp_async_wait<1>();                        // V of this page has landed
        __syncwarp();
#pragma unroll
        for (int run = 0; run < 4; ++run) {
            if (run * 16 < nv) {
                uint32_t pf[NB][2];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    pf[nb][0] = movm_trans(pack_bf16(s[nb][run][0], s[nb][run][1]));
                    pf[nb][1] = movm_trans(pack_bf16(s[nb][run][2], s[nb][run][3]));
                }
                uint32_t xs[2][2][NG / 2], vs[2][NG], vb[2][NG];       // codes by (h, j): two keys side by side; pairs of scales and of bases
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const uint8_t* at = vbuf + run * 8 * D + hh * 4 * D + lane * (D / 8);
                    const int key = run * 16 + hh * 8 + 2 * t;
                    const uint8_t* ps = vbuf + 32 * D + key * (D / 8);
                    uint32_t pa[2][NG];
                    if (D == 128) {
                        const uint4 v = *reinterpret_cast<const uint4*>(at);
                        xs[hh][0][0] = __byte_perm(v.x, v.z, 0x5410);
                        xs[hh][0][NG / 2 - 1] = __byte_perm(v.x, v.z, 0x7632);
                        xs[hh][1][0] = __byte_perm(v.y, v.w, 0x5410);
                        xs[hh][1][NG / 2 - 1] = __byte_perm(v.y, v.w, 0x7632);
                        *reinterpret_cast<uint4*>(&pa[0][0]) = *reinterpret_cast<const uint4*>(ps);
                        *reinterpret_cast<uint4*>(&pa[1][0]) = *reinterpret_cast<const uint4*>(ps + 16);
                    } else {
                        const uint2 v = *reinterpret_cast<const uint2*>(at);
                        xs[hh][0][0] = __byte_perm(v.x, v.y, 0x5410);
                        xs[hh][1][0] = __byte_perm(v.x, v.y, 0x7632);
                        *reinterpret_cast<uint2*>(&pa[0][0]) = *reinterpret_cast<const uint2*>(ps);
                        *reinterpret_cast<uint2*>(&pa[1][0]) = *reinterpret_cast<const uint2*>(ps + 8);
                    }
                    if (nv < KV4_PAGE) {           // what lies behind the last key may be anything: it must not meet a probability of zero as NaN
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            if (key + e >= nv)
#pragma unroll
                                for (int grp = 0; grp < NG; ++grp) pa[e][grp] = 0;
                    }
#pragma unroll
                    for (int grp = 0; grp < NG; ++grp) {
                        vs[hh][grp] = __byte_perm(pa[0][grp], pa[1][grp], 0x5410);
                        vb[hh][grp] = __byte_perm(pa[0][grp], pa[1][grp], 0x7632);
                    }
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const int grp = i >> 1, half = i >> 2, sh = 4 * (i & 3);
                    const uint32_t a0 = dequant2(codes128(xs[0][0][half], sh), vs[0][grp], vb[0][grp]);
                    const uint32_t a1 = dequant2(codes128(xs[0][1][half], sh), vs[0][grp], vb[0][grp]);
                    const uint32_t a2 = dequant2(codes128(xs[1][0][half], sh), vs[1][grp], vb[1][grp]);
                    const uint32_t a3 = dequant2(codes128(xs[1][1][half], sh), vs[1][grp], vb[1][grp]);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) mma_bf16(o[nb][i], a0, a1, a2, a3, pf[nb][0], pf[nb][1]);
                }
            }
        }
        __syncwarp();                              // every lane has read V
        fetch(1, id_next, nv_next);
        id = id_next;
        nv = nv_next;
    }
    cp_async_wait<0>();

    // ---- put the warps together: maxima and sums, then the outputs through shared memory
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) l[nb][e] += __shfl_xor_sync(0xffffffffu, l[nb][e], w);
            if (g == 0) warp_stat[warp][nb * 8 + 2 * t + e] = make_float2(m[nb][e], l[nb][e]);
        }
    __syncthreads();                               // also: every warp is done with its buffers
    float* osum = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        float top[2] = {-INFINITY, -INFINITY}, f[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int w = 0; w < DK_WARPS; ++w) top[e] = fmaxf(top[e], warp_stat[w][nb * 8 + 2 * t + e].x);
            f[e] = m[nb][e] == -INFINITY ? 0.f : ex2_ftz(m[nb][e] - top[e]);
        }
        float* to = osum + ((size_t)warp * 8 * NB + nb * 8 + 2 * t) * (D + 4) + g;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) to[(c & 1) * (D + 4) + i * 16 + (c >> 1) * 8] = f[c & 1] == 0.f ? 0.f : o[nb][i][c] * f[c & 1];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 8 * NB * D; i += DK_WARPS * 32) {
        const int q = i / D, d = i - q * D;
        if (head0 + q >= x.G) break;
        float top = -INFINITY, sum = 0.f, acc = 0.f;
#pragma unroll
        for (int w = 0; w < DK_WARPS; ++w) top = fmaxf(top, warp_stat[w][q].x);
#pragma unroll
        for (int w = 0; w < DK_WARPS; ++w) {
            const float2 st = warp_stat[w][q];
            if (st.y != 0.f) sum = fmaf(st.y, ex2_ftz(st.x - top), sum);      // 0: the warp had no keys
            acc += osum[((size_t)w * 8 * NB + q) * (D + 4) + d];
        }
        if (x.n_split == 1) {
            const __nv_bfloat16 v = __float2bfloat16_rn(n_page == 0 || sum == 0.f ? 0.f : acc / sum);
            x.O[((size_t)bh * x.G + head0 + q) * D + d] = __bfloat16_as_ushort(v);
        } else {
            const size_t at = ((size_t)unit * x.n_split + sp) * 8 * NB + q;
            x.part[at * D + d] = acc;
            if (d == 0) x.stats[at] = make_float2(top, sum);
        }
    }
}

// One block per (request, query head), thread = d: O = sum_c 2^(m_c - m) O_c / sum_c 2^(m_c - m) l_c over the splits in use.
template <int D>
__global__ void __launch_bounds__(D) k_attn_join_kv4(const DecodeKv4Args x, int heads) {
    dep_wait();
    const int q = blockIdx.x % x.G, bh = blockIdx.x / x.G, b = bh / x.H_kv, d = threadIdx.x;
    const int r = x.row ? x.row[b] : b;
    const int len = r >= 0 && r < x.n_rows ? min(max(x.len[r], 0), x.max_pages * KV4_PAGE) : 0;
    const int in_use = splits_in_use((len + KV4_PAGE - 1) / KV4_PAGE, x.n_split);
    const size_t at = ((size_t)(bh * x.h_blocks + q / heads) * x.n_split) * heads + q % heads;
    float m = -INFINITY;
    for (int c = 0; c < in_use; ++c) m = fmaxf(m, __ldcg(&x.stats[at + (size_t)c * heads]).x);
    float num = 0.f, den = 0.f;
#pragma unroll 4
    for (int c = 0; c < in_use; ++c) {
        const float2 st = __ldcg(&x.stats[at + (size_t)c * heads]);
        const float v = __ldcg(&x.part[(at + (size_t)c * heads) * D + d]);
        if (st.y != 0.f) {
            const float w = ex2_ftz(st.x - m);
            num = fmaf(w, v, num);
            den = fmaf(w, st.y, den);
        }
    }
    x.O[((size_t)bh * x.G + q) * D + d] = __bfloat16_as_ushort(__float2bfloat16_rn(den == 0.f ? 0.f : num / den));
}

// Heads of a block (8 or 16 rows of the MMA's N side), blocks per KV head, splits per unit - from the shape alone, so that the
// workspace can be sized without a device.  Splits: enough blocks for four rounds of two blocks on each of 148 SMs, none below DK_WARPS pages.
struct DecodeKv4Shape {
    int heads, h_blocks, n_split;
    long long units;
};
static bool decode_kv4_shape(long long B, int H_q, int H_kv, int D, int max_pages, DecodeKv4Shape* s) {
    if (B < 1 || H_kv < 1 || H_kv > 1024 || H_q < H_kv || H_q % H_kv || (D != 64 && D != 128) || max_pages < 1 || max_pages >= (1 << 25)) return false;
    const int G = H_q / H_kv;
    if (G > 1024) return false;
    s->heads = G <= 8 ? 8 : 16;
    s->h_blocks = (G + s->heads - 1) / s->heads;
    s->units = B * H_kv * s->h_blocks;
    const long long want = std::max(1ll, 4 * 2 * 148 / s->units);
    s->n_split = (int)std::min<long long>(std::min<long long>(want, DK_MAXSPLIT), (max_pages + DK_WARPS - 1) / DK_WARPS);
    return s->units * s->n_split <= 0x7fffffffll && B * H_q <= 0x7fffffffll;
}

}  // namespace ag

using namespace ag;

extern "C" size_t ag_attention_decode_kv4_workspace(int B, int H_q, int H_kv, int D, int max_pages) {
    DecodeKv4Shape s;
    if (!decode_kv4_shape(B, H_q, H_kv, D, max_pages, &s) || s.n_split == 1) return 0;
    return (size_t)s.units * s.n_split * s.heads * (sizeof(float2) + sizeof(float) * D);
}

extern "C" ag_status attention_decode_kv4(const void* Q, const ag_kv4_pool* pool, const ag_kv4_table* table, const int32_t* row, void* O, int B, int H_q,
                                          void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!kv4_pool_ok(pool) || !kv4_table_ok(table) || B < 0) return AG_ERR_ARG;
    if (B == 0) return AG_OK;
    DecodeKv4Shape s;
    if (!Q || !O || (((uintptr_t)Q | (uintptr_t)O) & 15u) || ((uintptr_t)row & 3u) || !decode_kv4_shape(B, H_q, pool->H_kv, pool->D, table->max_pages, &s) ||
        (!row && B > table->n_rows))
        return AG_ERR_ARG;
    const size_t need = ag_attention_decode_kv4_workspace(B, H_q, pool->H_kv, pool->D, table->max_pages);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 15u) || workspace_bytes < need)) return AG_ERR_ARG;
    ag_status st = check_arch();
    if (st != AG_OK) return st;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    DecodeKv4Args x;
    memset(&x, 0, sizeof x);
    x.Q = (const uint16_t*)Q;
    x.O = (uint16_t*)O;
    x.pages = (const uint8_t*)pool->pages;
    x.page_of = table->page_of; x.len = table->len; x.row = row;
    x.n_pages = (int)pool->n_pages; x.H_kv = pool->H_kv; x.G = H_q / pool->H_kv;
    x.n_rows = table->n_rows; x.max_pages = table->max_pages;
    x.n_split = s.n_split; x.h_blocks = s.h_blocks;
    x.scale_log2e = 1.4426950408889634f / sqrtf((float)pool->D);
    if (need > 0) {
        x.stats = (float2*)workspace;
        x.part = (float*)((uint8_t*)workspace + (size_t)s.units * s.n_split * s.heads * sizeof(float2));
    }
    const bool wide = s.heads == 16;
    void (*kernel)(DecodeKv4Args) = pool->D == 128 ? (wide ? k_attn_decode_kv4<128, 2> : k_attn_decode_kv4<128, 1>)
                                                   : (wide ? k_attn_decode_kv4<64, 2> : k_attn_decode_kv4<64, 1>);
    const int smem = pool->D == 128 ? (wide ? dk_smem_bytes<128, 2>() : dk_smem_bytes<128, 1>()) : (wide ? dk_smem_bytes<64, 2>() : dk_smem_bytes<64, 1>());
    static std::atomic<unsigned long long> attr_done{0};
    const cudaError_t attr_err = once_per_device(attr_done, [] {
        cudaError_t e = cudaFuncSetAttribute(k_attn_decode_kv4<128, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, dk_smem_bytes<128, 1>());
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k_attn_decode_kv4<128, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, dk_smem_bytes<128, 2>());
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k_attn_decode_kv4<64, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, dk_smem_bytes<64, 1>());
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k_attn_decode_kv4<64, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, dk_smem_bytes<64, 2>());
        return e;
    });
    if (attr_err != cudaSuccess) return cuda_fail(attr_err);
    kernel<<<(unsigned)(s.units * s.n_split), DK_WARPS * 32, smem, stream>>>(x);
    AG_CUDA(cudaGetLastError());
    count_launch();
    if (s.n_split > 1) {
        cudaLaunchConfig_t cfg;
        memset(&cfg, 0, sizeof cfg);
        cfg.gridDim = dim3((unsigned)((long long)B * H_q));
        cfg.blockDim = dim3(pool->D);
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        AG_CUDA(cudaLaunchKernelEx(&cfg, pool->D == 128 ? k_attn_join_kv4<128> : k_attn_join_kv4<64>, x, s.heads));
        count_launch();
    }
    return AG_OK;
}
