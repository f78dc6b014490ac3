// Single-token attention over the paged 4-bit key/value cache (layout: kv4.cuh).
//
// Per request, KV head and page of 64 keys, with the code u and the pair (s, b) of every element (value s u + b), G query heads:
//     S[key][q]  = sum over groups of 32 d:  s (sum_d u q_d) + b (sum_d q_d)      m16n8k16 MMA (fp16): 16 keys x 8 heads x 16 d
//     P = 2^((S - max) log2 e / sqrt D)                                           running maximum and sum per warp
//     O[d][q]   += sum_key V[key][d] P[key][q]                                    m16n8k16 MMA (fp16): 16 d x 8 heads x 16 keys
// A code of K becomes an fp16 operand with one logic instruction: a nibble masked out of its word is the subnormal u 2^-24, or u 2^-20, and
// the MMA takes subnormals as they are.  The bases' part comes from an MMA against sums over q kept in three bf16 parts (24 bits),
// so scores carry no rounding besides the 32-bit sums.  A subnormal operand may count as 2^-14 when the MMA lines its products up, in steps of 2^-24 of 1024 q s:
// 2^-13 sum |q| s / sqrt D for a score at most.  Measured with pairs of keys: 2^-19 of that sum, for queries up to 10^4 and with one channel that outweighs the
// others; the codes shifted up to 2^-18 u (three more instructions a word) measured the same and took 137.4 instead of 131.2 us for the long rows below.
// Outputs would feel it, so V's codes are not taken this way.  V varies its scale along the contraction: its codes become 16 + u
// (0x4C00 | u << 6) and then s u + b with one multiply-add, in fp16 under a power of two that follows the largest value: off by at most half
// a step of b - 16 s and half a step of the value, 2^-11 (|v| + |b - 16 s|), some 2^-10 of the group's largest, or 2^-32 of the row's largest;
// P, times 2^10, is fp16 as well, off by half a step, 2^-11 of itself.  (An fp8 MMA would take the codes as they are, but mma.sync on this chip converts fp8 operands to fp16
// first: measured, slower than the above.)
//
// Memory: 1.25 D bytes per key and head, read once for every 16 heads of a group.  A byte costs about ten times the arithmetic instructions of a bf16 cache's, and those bound
// it: 60 % of the issue slots are used, no pipe is at its limit (logic 50 %, tensor 20), the rest are fixed latencies of four warps a scheduler.  4 requests of 131072 keys, 32 query heads on 8, D = 128:
// 131 us, 5.0 TB/s (0.77 of the measured copy); 128 requests of 200 to 1024 keys: 35 us, half of it until the first page is there and from the last on.  So
// the operands are unpacked in registers, straight into the MMA's fragments (for tcgen05.mma they would go on into tensor memory; not built).  Groups of 9 to 16 heads
// take one block an SM (70 us against 50 for up to 8, 4 x 32768 keys), each 16 heads more another pass (121 us for 32, 218 for 64).  The cache stores the codes in fragment order, so a warp's share of a
// page is read with conflict-free vector loads.
//
// Work: all pages of all (request, KV head) units in one line, cut into equal runs, one per warp, every warp of the launch resident at
// once (two blocks of eight warps per SM).  A warp walks its run alone - one buffer each for K and V, refilled by 16-byte asynchronous
// copies as soon as it has been read: K of the next page comes in during the softmax and V's products, V during the next page's scores, while
// the SM's other warps are in other phases.  Uneven lengths, few long requests and many short ones are the same case.  Warps of a block that
// share a unit put their parts together at the end (fragment order, in the buffers that are free by then); a unit that goes beyond a block is left in
// one part per block for a second kernel.
#include <string.h>

#include <algorithm>

#include "kv4.cuh"

namespace ag {

constexpr int DK_WARPS = 8;
constexpr int DK_THREADS = DK_WARPS * 32;
// parts of a unit that the joining block can add up side by side (block of 2 D NB threads by so many, at most 1024)
__host__ __device__ constexpr int dk_join_lanes(int D, int NB) { return NB * D * 2 * 4 > 1024 ? 2 : 4; }

struct DecodeKv4Args {
    const uint16_t* Q;            // [B][H_q][D]
    uint16_t* O;                  // [B][H_q][D]
    const uint8_t* pages;
    const int32_t *page_of, *len, *row;
    float4* part;                 // [slots][NB][D / 16][32 lanes]: outputs (normalised) in fragment order; slots: 2 per warp, 2 per block
    float2* stats;                // [slots][8 NB]: maximum (in units of log2), sum
    int2* crossing;               // [blocks]: the unit that begins in the block and goes on beyond it (-1: none), the blocks that it has
    int B, n_pages, H_kv, G, n_rows, max_pages, h_blocks, n_blocks;
    int aligned;                  // 1: block = unit (short rows, few units)
    float scale_log2e;
};
__device__ __forceinline__ void mma_bf16_new(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_new(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t movm_trans(uint32_t v) {      // 8 x 8 matrix of 16-bit elements, transposed across the warp
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t mask, uint32_t bits) {      // (a & mask) | bits in one instruction
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(a), "r"(mask), "r"(bits));
    return r;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ int row_tokens(const DecodeKv4Args& x, int b, int* row) {
    const int r = x.row ? x.row[b] : b;
    *row = r;
    return r >= 0 && r < x.n_rows ? min(max(x.len[r], 0), x.max_pages * KV4_PAGE) : 0;
}
__device__ __forceinline__ int pages_of(int tokens) { return (tokens + KV4_PAGE - 1) / KV4_PAGE; }
// blocks that the line is cut for: at least a page for every warp
__device__ __forceinline__ int blocks_of(const DecodeKv4Args& x, long long total) { return (int)min((long long)x.n_blocks, (total + DK_WARPS - 1) / DK_WARPS); }
// the warp whose run holds place `at` of the line: run w begins at total * w / n
__device__ __forceinline__ int run_holding(long long at, long long total, int n) { return (int)(((at + 1) * n - 1) / total); }

// f a + g b, where a factor of zero means "not there", whatever stands beside it
__device__ __forceinline__ float weighted(float f, float a, float g, float b) { return (f == 0.f ? 0.f : f * a) + (g == 0.f ? 0.f : g * b); }
// Parts carry normalised outputs (no larger than the values, whatever the sums): a part with maximum pm and sum pl joins what there is (m, l), f and g being
// the shares of the outputs so far and of the part's.  pl = 0: a part without keys, g = 0.
__device__ __forceinline__ void join_weights(float& m, float& l, float pm, float pl, float& f, float& g) {
    const float top = fmaxf(m, pm);
    f = l == 0.f ? 0.f : m == top ? l : ex2_ftz(m - top) * l;
    g = pl == 0.f ? 0.f : pm == top ? pl : ex2_ftz(pm - top) * pl;
    l = f + g;
    const float r = l == 0.f ? 0.f : 1.f / l;
    f *= r;
    g *= r;
    m = pl == 0.f ? m : top;
}

// what a part with maximum pm and sum pl counts beside a maximum of `top`
__device__ __forceinline__ float part_weight(float pm, float pl, float top) { return pl == 0.f ? 0.f : pm == top ? pl : ex2_ftz(pm - top) * pl; }

// Where a warp is in the line of pages, apart from the page itself: needed once a page or once a unit, so it does not take registers.
// Every lane writes the same values.
struct WarpWalk {
    long long unit_begin, now_begin;               // place of the first page of the unit to be fetched from next / of the unit in hand
    int b, hh, len, row, now_unit, now_pages;
};

template <int D, int NB>
constexpr int dk_smem_bytes() { return DK_WARPS * (kv4_head_bytes(D) + NB * 8 * D * 2); }      // a head's page and a block of queries for each warp

template <int D, int NB>
__global__ void __launch_bounds__(DK_THREADS, NB == 1 ? 2 : 1) k_attn_decode_kv4(const DecodeKv4Args x) {
    constexpr int NG = D / 32;                     // groups of a row
    constexpr int MT = D / 16;                     // tiles of 16 d
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long before[DK_THREADS + 1];   // pages (of one KV head) in front of the share of requests that thread i counts
    __shared__ long long warp_sum[DK_WARPS];
    __shared__ int tokens_of[DK_THREADS], row_of[DK_THREADS];      // of the requests, up to DK_THREADS of them
    __shared__ int slot_unit[2 * DK_WARPS];        // units that a warp has only a part of: one that began before its run, one that goes on behind it
    __shared__ int slot_ends[2 * DK_WARPS];        // bit 0: the part includes the unit's last page; bit 1: it lies in the workspace, not in the warp's buffer
    __shared__ __align__(16) float2 slot_stats[2 * DK_WARPS][8 * NB];
    __shared__ float2 joint_stats[2 * DK_WARPS][8 * NB];           // of the unit that a part belongs to, over the block's parts
    __shared__ __align__(8) float slot_weight[2 * DK_WARPS][8 * NB];
    __shared__ WarpWalk walk[DK_WARPS];
    __shared__ long long line[2];                  // all pages of the line; the block's first place: needed again at the end, so they do not take registers
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    dep_wait();
    dep_release();

    // ---- this block's run, cut into the warps' runs: places of the line of pages; order: request, KV head (and block of query heads), page
    const int heads = x.H_kv * x.h_blocks;
    const int per = (x.B + DK_THREADS - 1) / DK_THREADS;
    long long total = 0, block_begin, block_end, first_unit_begin = 0;
    int b, hh = 0, p = 0, np, len, row;     // request b, KV head and block hh, page p of np
    if (x.aligned) {
        b = blockIdx.x / heads;
        hh = blockIdx.x - b * heads;
        len = row_tokens(x, b, &row);
        np = pages_of(len);
        block_begin = 0;
        block_end = np;
        if (np == 0) {
            for (int i = threadIdx.x; i < 8 * NB * D; i += DK_THREADS) {
                const int head = hh % x.h_blocks * 8 * NB + i / D;
                if (head < x.G) x.O[((size_t)(b * x.H_kv + hh / x.h_blocks) * x.G + head) * D + i % D] = 0;
            }
            return;
        }
    } else {
        long long n = 0;
        if (per == 1) {
            int r = 0, tokens = 0;
            if ((int)threadIdx.x < x.B) tokens = row_tokens(x, threadIdx.x, &r);
            tokens_of[threadIdx.x] = tokens;
            row_of[threadIdx.x] = r;
            n = pages_of(tokens);
        } else {
            for (int i = threadIdx.x * per, e = min(x.B, i + per), r; i < e; ++i) n += pages_of(row_tokens(x, i, &r));
        }
        long long inc = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += u;
        }
        if (lane == 31) warp_sum[warp] = inc;
        __syncthreads();
        long long add = 0;
#pragma unroll
        for (int w = 0; w < DK_WARPS; ++w) add += w < warp ? warp_sum[w] : 0;
        before[threadIdx.x] = add + inc - n;
        if (threadIdx.x == DK_THREADS - 1) before[DK_THREADS] = add + inc;
        __syncthreads();
        total = before[DK_THREADS] * heads;
        const int n_blocks = blocks_of(x, total);
        for (int i = blockIdx.x; i < x.B; i += gridDim.x) {         // requests without keys: zeros
            int r;
            if ((per > 1 ? row_tokens(x, i, &r) : tokens_of[i]) != 0) continue;
            uint4* out = reinterpret_cast<uint4*>(x.O + (size_t)i * x.H_kv * x.G * D);
            for (int k = threadIdx.x; k < x.H_kv * x.G * D / 8; k += DK_THREADS) out[k] = make_uint4(0, 0, 0, 0);
        }
        if ((int)blockIdx.x >= n_blocks) {
            if (threadIdx.x == 0) x.crossing[blockIdx.x] = make_int2(-1, 0);
            return;
        }
        block_begin = total * blockIdx.x / n_blocks;
        block_end = total * (blockIdx.x + 1) / n_blocks;
        b = 0;
        len = np = row = 0;
    }
    auto request = [&](int i, int* r) {            // tokens and row of request i (not in aligned launches)
        if (per > 1) return row_tokens(x, i, r);
        *r = row_of[i];
        return tokens_of[i];
    };
    if (threadIdx.x < 2 * DK_WARPS) slot_unit[threadIdx.x] = -1;
    if (threadIdx.x == 0) {
        line[0] = total;
        line[1] = block_begin;
    }
    __syncthreads();
    const long long begin = block_begin + (block_end - block_begin) * warp / DK_WARPS;
    int left = (int)(block_begin + (block_end - block_begin) * (warp + 1) / DK_WARPS - begin);

    uint8_t* kbuf = smem + warp * kv4_head_bytes(D);          // codes of K, then K's pairs
    uint8_t* vbuf = kbuf + 40 * D;
    uint8_t* qbuf = smem + DK_WARPS * kv4_head_bytes(D) + warp * (NB * 8 * D * 2);
    const uint32_t kbuf_a = smem_u32(kbuf), vbuf_a = smem_u32(vbuf), qbuf_a = smem_u32(qbuf);
    // copies the runs of 16 tokens that hold keys: codes (8 D bytes a run) and pairs (2 D bytes a run)
    auto fetch = [&](int which, const uint8_t* src, int nv) {
        if (nv > 0) {
            const uint32_t dst = which ? vbuf_a : kbuf_a;
            const uint8_t* codes = src + which * 32 * D + lane * 16;
            const uint8_t* pairs = src + 64 * D + which * 8 * D + lane * 16;
            if (nv > 48) {
#pragma unroll
                for (int j = 0; j < 32 * D / 512; ++j) cp_async16(dst + j * 512 + lane * 16, codes + j * 512);
#pragma unroll
                for (int j = 0; j < 8 * D / 512; ++j) cp_async16(dst + 32 * D + j * 512 + lane * 16, pairs + j * 512);
            } else {
                const int runs = (nv + 15) >> 4;
                for (int j = lane * 16; j < runs * 8 * D; j += 512) cp_async16(dst + j, codes + (j - lane * 16));
                for (int j = lane * 16; j < runs * 2 * D; j += 512) cp_async16(dst + 32 * D + j, pairs + (j - lane * 16));
            }
        }
        cp_async_commit();
    };

    // copies the query rows of KV head and block hh of request b
    auto fetch_q = [&](int b, int hh) {
        const int head0 = hh % x.h_blocks * 8 * NB, rows = min(x.G - head0, 8 * NB);
        const uint8_t* src = reinterpret_cast<const uint8_t*>(x.Q + (((size_t)b * x.H_kv + hh / x.h_blocks) * x.G + head0) * D);
        for (int j = lane * 16; j < rows * 2 * D; j += 512) cp_async16(qbuf_a + j, src + j);
    };

    // ---- the first page of the run
    if (x.aligned) {
        p = (int)begin;
    } else if (left > 0) {
        const long long at = begin / heads;
        int lo = 0, hi = DK_THREADS - 1;           // the last share that begins at or in front of it
        while (lo < hi) {
            const int m = (lo + hi + 1) >> 1;
            if (before[m] <= at) lo = m; else hi = m - 1;
        }
        b = lo * per;
        long long in_front = before[lo];
        while (true) {
            len = request(b, &row);
            np = pages_of(len);
            if (in_front + np > at) break;
            in_front += np;
            ++b;
        }
        const long long rest = begin - in_front * heads;
        hh = (int)(rest / np);
        p = (int)(rest - (long long)hh * np);
        first_unit_begin = begin - p;
    }
    WarpWalk* at = &walk[warp];
    at->unit_begin = first_unit_begin;
    at->b = b;
    at->hh = hh;
    at->len = len;
    at->row = row;
    __syncwarp();
    const int p_first = p;
    int id_batch = 0, id_first = -64;              // ids of pages id_first + lane of the row (reloaded as p leaves them)
    const uint8_t* src_next = nullptr;
    int nv_next = 0;
    auto locate = [&]() {                          // source and number of keys of page p
        if (p < id_first || p >= id_first + 32) {
            id_first = p;
            id_batch = p + lane < np ? x.page_of[(size_t)at->row * x.max_pages + p + lane] : -1;
        }
        const int id = __shfl_sync(0xffffffffu, id_batch, p - id_first);
        nv_next = id >= 0 && id < x.n_pages ? min(KV4_PAGE, at->len - p * KV4_PAGE) : 0;
        src_next = x.pages + ((size_t)(nv_next ? id : 0) * x.H_kv + at->hh / x.h_blocks) * kv4_head_bytes(D);
    };
    if (left > 0) {
        fetch_q(b, hh);                            // (in front of the pages, so as not to queue behind everybody's)
        cp_async_commit();
        locate();
        fetch(0, src_next, nv_next);
        fetch(1, src_next, nv_next);
    }

    uint32_t qb[NB][2];
    float unscale[NB][2];                          // log2 e / (c sqrt D) of heads 2 t and 2 t + 1
    float o[NB][MT][4];
    float m[NB][2], l[NB][2];
    int v_exp = 0;                                 // outputs are kept times 2^(13 - v_exp)
    bool fresh = true;                             // the page in hand is the first of a unit for this warp
    bool whole = p_first == 0;                     // this warp has had the unit from its first page
    // Where the outputs of a unit go.  Fragments have heads 2 t, 2 t + 1 of d = 16 i + g, + 8 in lane (g, t); transposed, head g of d = 16 i + 2 t, + 1, ...
    auto out_of = [&](int unit, int* head0) {
        const int bu = unit / heads, hu = unit - bu * heads;
        *head0 = hu % x.h_blocks * 8 * NB;
        return x.O + (((size_t)bu * x.H_kv + hu / x.h_blocks) * x.G + *head0 + g) * D + 2 * t;
    };
    auto write_fragment = [&](uint16_t* out, int head0, int nb, int i, float v0, float v1, float v2, float v3) {
        const uint32_t lo = movm_trans(pack_bf16(v0, v1)), hi = movm_trans(pack_bf16(v2, v3));
        if (head0 + nb * 8 + g < x.G) {
            *reinterpret_cast<uint32_t*>(out + nb * 8 * D + i * 16) = lo;
            *reinterpret_cast<uint32_t*>(out + nb * 8 * D + i * 16 + 8) = hi;
        }
    };
    while (left > 0) {
        const int nv = nv_next;
        if (fresh) {
            const int b_now = at->b, hh_now = at->hh;
            const int head0 = hh_now % x.h_blocks * 8 * NB;       // first query head of the block, of the KV head's G
            at->now_unit = b_now * heads + hh_now;
            at->now_pages = np;
            at->now_begin = at->unit_begin;
            cp_async_wait<2>();                    // the queries have landed
            __syncwarp();
            // ---- queries as B operands: q times a power of two c (the head's largest |q| between 2^14 and 2^15) in fp16, exact down to
            // 2^-24 of the largest.  Lane (g, t) holds head g, elements 32 grp + 8 t + {0, 4}, {1, 5}, {2, 6}, {3, 7}.  Even elements meet
            // 2^-24 u, odd ones, kept at a sixteenth, 2^-20 u (see the scores).  The bases meet the groups' sums of q, times 2^-24 c, 24 bits in
            // three bf16 parts.
            uint32_t qf[NB][NG][4];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int head = head0 + nb * 8 + g;
                float q[NG][8], top = 0.f;
#pragma unroll
                for (int grp = 0; grp < NG; ++grp) {
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (head < x.G) v = *reinterpret_cast<const uint4*>(qbuf + (nb * 8 + g) * D * 2 + grp * 64 + t * 16);
                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        q[grp][2 * i] = bf16_lo(w[i]);
                        q[grp][2 * i + 1] = bf16_hi(w[i]);
                        top = fmaxf(top, fmaxf(fabsf(q[grp][2 * i]), fabsf(q[grp][2 * i + 1])));
                    }
                }
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const uint32_t e = min(246u, 268u - (__float_as_uint(top) >> 23));        // exponent field of c
                const float c = __uint_as_float(e << 23);
                float total[NG];
#pragma unroll
                for (int grp = 0; grp < NG; ++grp) {
                    total[grp] = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        q[grp][i] *= c;
                        total[grp] += q[grp][i];
                        if (i & 1) q[grp][i] *= 0x1p-4f;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) qf[nb][grp][i] = pack_f16(q[grp][i], q[grp][i + 4]);
#pragma unroll
                    for (int w = 1; w < 4; w <<= 1) total[grp] += __shfl_xor_sync(0xffffffffu, total[grp], w);
                }
                // D = 128: k = 2 t, 2 t + 1 are groups 2 (t & 1), + 1 of part t / 2, k + 8 part 2 of them (t < 2); D = 64: both groups, part t
                const bool upper = D == 128 && (t & 1);
                const int part = D == 128 ? t >> 1 : t;
                uint32_t sums[3];                          // the lane's two groups, bf16 side by side
                float s0 = 0x1p-24f * (upper ? total[NG - 2] : total[0]), s1 = 0x1p-24f * (upper ? total[NG - 1] : total[1]);
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    sums[k] = pack_bf16(s0, s1);
                    s0 -= bf16_lo(sums[k]);
                    s1 -= bf16_hi(sums[k]);
                }
                qb[nb][0] = part == 0 ? sums[0] : part == 1 ? sums[1] : part == 2 ? sums[2] : 0u;
                qb[nb][1] = D == 128 && t < 2 ? sums[2] : 0u;
                const float f = x.scale_log2e * 0x1p24f * __uint_as_float((254u - e) << 23);
                unscale[nb][0] = __shfl_sync(0xffffffffu, f, 8 * t);
                unscale[nb][1] = __shfl_sync(0xffffffffu, f, 8 * t + 4);
            }
            __syncwarp();                          // every lane has read its rows; the operands take their place, and are fetched once a page
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int grp = 0; grp < NG; ++grp)
                    *reinterpret_cast<uint4*>(qbuf + ((nb * NG + grp) * 32 + lane) * 16) = make_uint4(qf[nb][grp][0], qf[nb][grp][1], qf[nb][grp][2], qf[nb][grp][3]);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int c = 0; c < 4; ++c) o[nb][i][c] = 0.f;
                m[nb][0] = m[nb][1] = -INFINITY;
                l[nb][0] = l[nb][1] = 0.f;
            }
            v_exp = -100;
        }
        cp_async_wait<1>();                        // K of this page has landed
        __syncwarp();
        // (the runs behind the last key are computed with the others: what they hold does not count, see below)
        float s[NB][4][4];
        if (nv > 0) {
            uint4 qf[NB][NG];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int grp = 0; grp < NG; ++grp) qf[nb][grp] = *reinterpret_cast<const uint4*>(qbuf + ((nb * NG + grp) * 32 + lane) * 16);
#pragma unroll
            for (int run = 0; run < 4; ++run) {
                uint32_t w[2][NG], sb[2][NG], bb[2];            // rows g and g + 8 of the run: codes, pairs, two groups' bases as A operands
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const uint8_t* at = kbuf + run * 8 * D + hh * 4 * D + lane * (D / 8);
                    const uint8_t* ps = kbuf + 32 * D + (run * 16 + hh * 8 + g) * (D / 8);
                    if (D == 128) {
                        *reinterpret_cast<uint4*>(&w[hh][0]) = *reinterpret_cast<const uint4*>(at);
                        *reinterpret_cast<uint4*>(&sb[hh][0]) = *reinterpret_cast<const uint4*>(ps);
                        const uint2 two = *reinterpret_cast<const uint2*>(ps + (t & 1) * 8);
                        bb[hh] = __byte_perm(two.x, two.y, 0x7632);
                    } else {
                        *reinterpret_cast<uint2*>(&w[hh][0]) = *reinterpret_cast<const uint2*>(at);
                        *reinterpret_cast<uint2*>(&sb[hh][0]) = *reinterpret_cast<const uint2*>(ps);
                        bb[hh] = __byte_perm(sb[hh][0], sb[hh][1], 0x7632);
                    }
                }
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) mma_bf16_new(s[nb][run], bb[0], bb[1], D == 128 ? bb[0] : 0u, D == 128 ? bb[1] : 0u, qb[nb][0], qb[nb][1]);
#pragma unroll
                for (int grp = 0; grp < NG; ++grp) {
                    const float s0 = bf16_lo(sb[0][grp]), s1 = bf16_lo(sb[1][grp]);
                    // a nibble by itself is a subnormal fp16, u 2^-24 or (one nibble up) u 2^-20
                    uint32_t a[2][4];
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh) {
                        const uint32_t w8 = w[hh][grp] >> 8;
                        a[hh][0] = w[hh][grp] & 0x000f000fu;
                        a[hh][1] = w[hh][grp] & 0x00f000f0u;
                        a[hh][2] = w8 & 0x000f000fu;
                        a[hh][3] = w8 & 0x00f000f0u;
                    }
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        float acc[4];
                        mma_f16_new(acc, a[0][0], a[1][0], a[0][1], a[1][1], qf[nb][grp].x, qf[nb][grp].y);
                        mma_f16(acc, a[0][2], a[1][2], a[0][3], a[1][3], qf[nb][grp].z, qf[nb][grp].w);
                        s[nb][run][0] = fmaf(s0, acc[0], s[nb][run][0]);
                        s[nb][run][1] = fmaf(s0, acc[1], s[nb][run][1]);
                        s[nb][run][2] = fmaf(s1, acc[2], s[nb][run][2]);
                        s[nb][run][3] = fmaf(s1, acc[3], s[nb][run][3]);
                    }
                }
            }
        }
        __syncwarp();                              // every lane has read K
        // ---- on to the next page: same unit, next head, next request that has any
        // (the queries' operands have been read as well)
        const bool ends = p + 1 == np;
        --left;
        nv_next = 0;
        if (left > 0) {
            ++p;
            if (ends) {
                int bn = at->b, hn = at->hh + 1, rn, ln;
                const long long next_begin = at->unit_begin + np;
                __syncwarp();                      // every lane has read them
                at->unit_begin = next_begin;
                p = 0;
                if (hn == heads) {
                    hn = 0;
                    do {
                        ++bn;
                        ln = request(bn, &rn);
                        np = pages_of(ln);
                    } while (np == 0);
                    id_first = -64;
                    at->b = bn;
                    at->len = ln;
                    at->row = rn;
                }
                at->hh = hn;
                __syncwarp();
                fetch_q(at->b, hn);
            }
            locate();
        }
        cp_async_commit();
        fetch(0, src_next, nv_next);
        if (nv > 0) {
            // ---- softmax, with the running maximum in the scores' own units; keys past the end count as -inf
            if (nv < KV4_PAGE) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int run = 0; run < 4; ++run)
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            if (run * 16 + g + (c >> 1) * 8 >= nv) s[nb][run][c] = -INFINITY;
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float top[2] = {m[nb][0], m[nb][1]};
#pragma unroll
                for (int run = 0; run < 4; ++run)
#pragma unroll
                    for (int c = 0; c < 4; ++c) top[c & 1] = fmaxf(top[c & 1], s[nb][run][c]);
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int w = 4; w < 32; w <<= 1) top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], w));
                if (__any_sync(0xffffffffu, top[0] != m[nb][0] || top[1] != m[nb][1])) {
                    float f[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        f[e] = top[e] == m[nb][e] ? 1.f : ex2_ftz((m[nb][e] - top[e]) * unscale[nb][e]);
                        l[nb][e] *= f[e];
                        m[nb][e] = top[e];
                    }
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int c = 0; c < 4; ++c) o[nb][i][c] *= f[c & 1];
                }
                float ref[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) ref[e] = m[nb][e] == -INFINITY ? 0.f : fmaf(m[nb][e], unscale[nb][e], -10.f);      // P is kept times 2^10: fp16 then holds it down to 2^-34
#pragma unroll
                for (int run = 0; run < 4; ++run)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        s[nb][run][c] = ex2_ftz(fmaf(s[nb][run][c], unscale[nb][c & 1], -ref[c & 1]));
                        l[nb][c & 1] += s[nb][run][c];
                    }
            }
        }
        cp_async_wait<2>();                        // V of this page has landed
        __syncwarp();
        if (nv > 0) {
            // The pairs of two keys side by side (s, s') and (c, c'), c = b - 16 s, in fp16 times 2^(13 - v_exp): |b| + 31 s, the largest a value
            // can be, stays below 2^15.  Lane = pair of keys; in place.  What lies behind the last key may be anything and becomes zero.
            uint32_t* pairs = reinterpret_cast<uint32_t*>(vbuf + 32 * D) + lane * 2 * NG;
            uint32_t w[2][NG];
            float top = 0.f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (D == 128) *reinterpret_cast<uint4*>(&w[e][0]) = *reinterpret_cast<const uint4*>(pairs + e * NG);
                else *reinterpret_cast<uint2*>(&w[e][0]) = *reinterpret_cast<const uint2*>(pairs + e * NG);
#pragma unroll
                for (int grp = 0; grp < NG; ++grp) {
                    if (2 * lane + e >= nv) w[e][grp] = 0u;
                    top = fmaxf(top, fmaf(31.f, fabsf(bf16_lo(w[e][grp])), fabsf(bf16_hi(w[e][grp]))));
                }
            }
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            const int e_top = max(-100, (int)(__float_as_uint(top) >> 23) - 127);
            if (e_top > v_exp + 1) {               // larger values than before: the outputs so far move to the new exponent (the same for all lanes)
                const float f = v_exp < e_top - 126 ? 0.f : __uint_as_float((uint32_t)(127 + v_exp - e_top) << 23);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int c = 0; c < 4; ++c) o[nb][i][c] *= f;
                v_exp = e_top;
            }
            const float k = __uint_as_float((uint32_t)(127 + 13 - v_exp) << 23);
            uint32_t sc[2][NG];
#pragma unroll
            for (int grp = 0; grp < NG; ++grp) {
                const float s0 = bf16_lo(w[0][grp]) * k, s1 = bf16_lo(w[1][grp]) * k;
                sc[0][grp] = pack_f16(s0, s1);
                sc[1][grp] = pack_f16(fmaf(bf16_hi(w[0][grp]), k, -16.f * s0), fmaf(bf16_hi(w[1][grp]), k, -16.f * s1));
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (D == 128) *reinterpret_cast<uint4*>(pairs + e * NG) = *reinterpret_cast<const uint4*>(&sc[e][0]);
                else *reinterpret_cast<uint2*>(pairs + e * NG) = *reinterpret_cast<const uint2*>(&sc[e][0]);
            }
            __syncwarp();
#pragma unroll
            for (int run = 0; run < 4; ++run) {
                uint32_t pf[NB][2];                // probabilities as B operands
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int e = 0; e < 2; ++e) pf[nb][e] = movm_trans(pack_f16(s[nb][run][2 * e], s[nb][run][2 * e + 1]));
                uint32_t xs[2][2][NG / 2], vs[2][NG], vc[2][NG];       // codes by (h, j): two keys side by side; pairs of scales and of bases
#pragma unroll
                for (int hh2 = 0; hh2 < 2; ++hh2) {
                    const uint8_t* at = vbuf + run * 8 * D + hh2 * 4 * D + lane * (D / 8);
                    const uint8_t* ps = vbuf + 32 * D + (run * 8 + hh2 * 4 + t) * (D / 4);
                    if (D == 128) {
                        const uint4 v = *reinterpret_cast<const uint4*>(at);
                        xs[hh2][0][0] = __byte_perm(v.x, v.z, 0x5410);
                        xs[hh2][0][NG / 2 - 1] = __byte_perm(v.x, v.z, 0x7632);
                        xs[hh2][1][0] = __byte_perm(v.y, v.w, 0x5410);
                        xs[hh2][1][NG / 2 - 1] = __byte_perm(v.y, v.w, 0x7632);
                        *reinterpret_cast<uint4*>(&vs[hh2][0]) = *reinterpret_cast<const uint4*>(ps);
                        *reinterpret_cast<uint4*>(&vc[hh2][0]) = *reinterpret_cast<const uint4*>(ps + 16);
                    } else {
                        const uint2 v = *reinterpret_cast<const uint2*>(at);
                        xs[hh2][0][0] = __byte_perm(v.x, v.y, 0x5410);
                        xs[hh2][1][0] = __byte_perm(v.x, v.y, 0x7632);
                        *reinterpret_cast<uint2*>(&vs[hh2][0]) = *reinterpret_cast<const uint2*>(ps);
                        *reinterpret_cast<uint2*>(&vc[hh2][0]) = *reinterpret_cast<const uint2*>(ps + 8);
                    }
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    // fp16 0x4C00 | u << 6 = 16 + u, and (16 + u) s + c = s u + b, rounded once
                    const int grp = i >> 1, half = i >> 2, k = i & 3;
                    uint32_t a[2][2];
#pragma unroll
                    for (int hh2 = 0; hh2 < 2; ++hh2)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const uint32_t w = xs[hh2][j][half];
                            const uint32_t c = and_or(k == 0 ? w << 6 : k == 1 ? w << 2 : k == 2 ? w >> 2 : w >> 6, 0x03c003c0u, 0x4c004c00u);
                            a[hh2][j] = fma_f16x2(c, vs[hh2][grp], vc[hh2][grp]);
                        }
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) mma_f16(o[nb][i], a[0][0], a[0][1], a[1][0], a[1][1], pf[nb][0], pf[nb][1]);
                }
            }
        }
        __syncwarp();                              // every lane has read V
        fetch(1, src_next, nv_next);

        // ---- the end of the unit, or of this warp's share of it
        if (ends || left == 0) {
            const float unexp = __uint_as_float((uint32_t)(127 - 13 + v_exp) << 23);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int w = 4; w < 32; w <<= 1) l[nb][e] += __shfl_xor_sync(0xffffffffu, l[nb][e], w);
                    m[nb][e] = m[nb][e] == -INFINITY ? -INFINITY : m[nb][e] * unscale[nb][e];      // in units of log2 from here on
                }
                // normalised here, while the outputs are in their own exponent: the sum of p v itself may be beyond 32 bits
                const float r[2] = {l[nb][0] == 0.f ? 0.f : unexp / l[nb][0], l[nb][1] == 0.f ? 0.f : unexp / l[nb][1]};
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int c = 0; c < 4; ++c) o[nb][i][c] *= r[c & 1];
            }
            const int unit = at->now_unit;
            if (whole && ends) {
                int head0;
                uint16_t* out = out_of(unit, &head0);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int i = 0; i < MT; ++i) write_fragment(out, head0, nb, i, o[nb][i][0], o[nb][i][1], o[nb][i][2], o[nb][i][3]);
            } else {
                // a part: into the warp's own buffer when that has been read for the last time (64 D of its 80 D bytes, or half of it)
                const int slot = 2 * warp + (whole ? 1 : 0);
                float4* to = left == 0 ? reinterpret_cast<float4*>(kbuf) : x.part + (2 * DK_WARPS * (size_t)blockIdx.x + slot) * NB * MT * 32;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    if (g == 0) *reinterpret_cast<float4*>(&slot_stats[slot][nb * 8 + 2 * t]) = make_float4(m[nb][0], l[nb][0], m[nb][1], l[nb][1]);
#pragma unroll
                    for (int i = 0; i < MT; ++i) to[(nb * MT + i) * 32 + lane] = make_float4(o[nb][i][0], o[nb][i][1], o[nb][i][2], o[nb][i][3]);
                }
                if (lane == 0) {
                    slot_unit[slot] = unit;
                    slot_ends[slot] = (ends ? 1 : 0) | (left == 0 ? 0 : 2);
                }
            }
            if (left == 0 && warp == DK_WARPS - 1 && lane == 0 && !x.aligned) {      // the block's last page (no warp behind this one's has any)
                int2 cross = make_int2(-1, 0);
                const long long all = line[0];
                if (!ends && at->now_begin >= line[1])
                    cross = make_int2(unit, run_holding(at->now_begin + at->now_pages - 1, all, blocks_of(x, all)) - (int)blockIdx.x + 1);
                x.crossing[blockIdx.x] = cross;
            }
            whole = true;                          // whatever comes next begins in this warp's run
        }
        fresh = ends;
    }
    cp_async_wait<0>();

    // ---- parts of units that several warps have: O = sum_c w_c O_c / sum_c w_c, w_c = 2^(m_c - m) l_c, over the parts c with keys that count.  The slots
    // are in the order of the line, so a unit's parts are neighbours.  The warps share the work by fragments.
    __syncthreads();
    const int slot_u = lane < 2 * DK_WARPS ? slot_unit[lane] : -1;
    const unsigned there = __ballot_sync(0xffffffffu, slot_u >= 0), in_front = there & ((1u << lane) - 1u);
    const unsigned with_end = __ballot_sync(0xffffffffu, slot_u >= 0 && (slot_ends[lane % (2 * DK_WARPS)] & 1));
    const unsigned far = __ballot_sync(0xffffffffu, slot_u >= 0 && (slot_ends[lane % (2 * DK_WARPS)] & 2));
    const int prev_u = __shfl_sync(0xffffffffu, slot_u, in_front ? 31 - __clz(in_front) : 0);
    const unsigned firsts = __ballot_sync(0xffffffffu, slot_u >= 0 && !(in_front && prev_u == slot_u));
    const unsigned same = __match_any_sync(0xffffffffu, slot_u) & there;            // the parts of the lane's slot's unit
    static_assert(2 * DK_WARPS * 8 * NB <= DK_THREADS, "a thread for every part and head");
    {
        const int slot = threadIdx.x / (8 * NB), head = threadIdx.x % (8 * NB);
        const unsigned parts = __shfl_sync(0xffffffffu, same, slot % (2 * DK_WARPS));
        if (slot < 2 * DK_WARPS && (parts >> slot & 1)) {
            float top = -INFINITY, sum = 0.f;
            for (unsigned c = parts; c; c &= c - 1) {
                const float2 st = slot_stats[__ffs(c) - 1][head];
                if (st.y != 0.f) top = fmaxf(top, st.x);
            }
            for (unsigned c = parts; c; c &= c - 1) {
                const float2 st = slot_stats[__ffs(c) - 1][head];
                sum += part_weight(st.x, st.y, top);
            }
            const float2 st = slot_stats[slot][head];
            slot_weight[slot][head] = sum == 0.f ? 0.f : part_weight(st.x, st.y, top) / sum;
            joint_stats[slot][head] = make_float2(top, sum);
        }
    }
    __syncthreads();
    const int n_items = __popc(firsts) * MT, k1 = n_items * (warp + 1) / DK_WARPS;       // the fragments of all units in one line, cut into equal runs
    for (int k = n_items * warp / DK_WARPS; k < k1;) {
        unsigned rest = firsts;
        for (int q = k / MT; q; --q) rest &= rest - 1;
        const int own = __ffs(rest) - 1, unit = __shfl_sync(0xffffffffu, slot_u, own), i0 = k % MT, i1 = min(MT, i0 + k1 - k);
        k += i1 - i0;
        const unsigned parts = __ballot_sync(0xffffffffu, slot_u == unit);
        const bool starts = (own & 1) || x.aligned;
        const size_t joint = 2 * DK_WARPS * (size_t)x.n_blocks + 2 * (size_t)blockIdx.x + (starts ? 1 : 0);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            float4 v[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            for (unsigned c = parts; c; c &= c - 1) {
                const int slot = __ffs(c) - 1;
                const float2 w = *reinterpret_cast<const float2*>(&slot_weight[slot][nb * 8 + 2 * t]);     // (a weight of zero: whatever stands there)
                const float4* from = (far >> slot & 1 ? x.part + (2 * DK_WARPS * (size_t)blockIdx.x + slot) * NB * MT * 32
                                                      : reinterpret_cast<const float4*>(smem + (slot >> 1) * kv4_head_bytes(D))) + nb * MT * 32 + lane;
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    if (i < i0 || i >= i1) continue;
                    const float4 u = from[i * 32];
                    v[i].x += w.x == 0.f ? 0.f : w.x * u.x;
                    v[i].y += w.y == 0.f ? 0.f : w.y * u.y;
                    v[i].z += w.x == 0.f ? 0.f : w.x * u.z;
                    v[i].w += w.y == 0.f ? 0.f : w.y * u.w;
                }
            }
            if (starts && (with_end & parts)) {
                int head0;
                uint16_t* out = out_of(unit, &head0);
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    if (i >= i0 && i < i1) write_fragment(out, head0, nb, i, v[i].x, v[i].y, v[i].z, v[i].w);
            } else {
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    if (i >= i0 && i < i1) x.part[((joint * NB + nb) * MT + i) * 32 + lane] = v[i];
                if (i0 == 0 && lane < 8) x.stats[joint * 8 * NB + nb * 8 + lane] = joint_stats[own][nb * 8 + lane];
            }
        }
    }
}

// Block i joins the unit that began in block i of the main kernel and went on beyond it, thread (j, y): fragment j of the output, parts y,
// y + blockDim.y, ...:  O = sum_c w_c O_c / sum_c w_c, w_c = 2^(m_c - m) l_c.  A part without a key that counts has m_c = -inf, l_c = 0 and is left out.
template <int D, int NB>
__global__ void __launch_bounds__(NB * D * 2 * dk_join_lanes(D, NB)) k_attn_join_kv4(const DecodeKv4Args x) {
    constexpr int MT = D / 16, NF = NB * MT * 32, LANES = dk_join_lanes(D, NB);
    __shared__ float4 acc[LANES - 1][NF];
    __shared__ float4 stat[LANES - 1][NF];
    dep_wait();
    const int j = threadIdx.x, y = threadIdx.y, lane = j & 31, g = lane >> 2, t = lane & 3, i = (j >> 5) % MT, nb = (j >> 5) / MT;
    const int2 pc = x.crossing[blockIdx.x];
    if (pc.x < 0) return;
    const int heads = x.H_kv * x.h_blocks, b = pc.x / heads, hh = pc.x - b * heads;
    const int head = hh % x.h_blocks * 8 * NB + nb * 8 + 2 * t;
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    auto join = [&](const float4& st, const float4& u) {
        float f0, f1, g0, g1;
        join_weights(m0, l0, st.x, st.y, f0, g0);
        join_weights(m1, l1, st.z, st.w, f1, g1);
        v.x = weighted(f0, v.x, g0, u.x);
        v.y = weighted(f1, v.y, g1, u.y);
        v.z = weighted(f0, v.z, g0, u.z);
        v.w = weighted(f1, v.w, g1, u.w);
    };
    if (head < x.G) {
        auto slot = [&](int c) { return 2 * DK_WARPS * (size_t)x.n_blocks + 2 * (size_t)(blockIdx.x + c) + (c == 0 ? 1 : 0); };
#pragma unroll 4
        for (int c = y; c < pc.y; c += blockDim.y) {       // (maximum, sum and outputs in passes of their own took 58 us instead of 55.6 for 131072 keys)
            const float4 st = __ldcg(reinterpret_cast<const float4*>(&x.stats[slot(c) * 8 * NB + nb * 8 + 2 * t]));
            const float4 u = __ldcg(&x.part[((slot(c) * NB + nb) * MT + i) * 32 + lane]);
            join(st, u);
        }
    }
    if (y > 0) {
        acc[y - 1][j] = v;
        stat[y - 1][j] = make_float4(m0, l0, m1, l1);
    }
    if (blockDim.y > 1) __syncthreads();
    if (y > 0 || head >= x.G) return;
    for (int k = 0; k < (int)blockDim.y - 1; ++k) {
        join(stat[k][j], acc[k][j]);
    }
    uint16_t* out = x.O + ((size_t)(b * x.H_kv + hh / x.h_blocks) * x.G + head) * D + 16 * i + g;
    out[0] = __bfloat16_as_ushort(__float2bfloat16_rn(v.x));
    out[8] = __bfloat16_as_ushort(__float2bfloat16_rn(v.z));
    if (head + 1 < x.G) {
        out[D] = __bfloat16_as_ushort(__float2bfloat16_rn(v.y));
        out[D + 8] = __bfloat16_as_ushort(__float2bfloat16_rn(v.w));
    }
}

// Blocks of query heads (8 or 16 rows of the MMA's N side), warps - from the shape alone, so that the workspace can be sized without a
// device.  Every warp is resident at once: 148 SMs times two blocks of eight warps with 8 heads, one with 16 (255 registers a thread).
struct DecodeKv4Shape {
    int nb, h_blocks, n_blocks, aligned;
    long long units;
    size_t slots() const { return (2 * DK_WARPS + 2) * (size_t)n_blocks; }
};
static bool decode_kv4_shape(long long B, int H_q, int H_kv, int D, int max_pages, DecodeKv4Shape* s) {
    if (B < 1 || H_kv < 1 || H_kv > 1024 || H_q < H_kv || H_q % H_kv || (D != 64 && D != 128) || max_pages < 1 || max_pages >= (1 << 25)) return false;
    const int G = H_q / H_kv;
    if (G > 1024) return false;
    s->nb = G <= 8 ? 1 : 2;
    s->h_blocks = (G + 8 * s->nb - 1) / (8 * s->nb);
    s->units = B * H_kv * s->h_blocks;
    const int most = s->nb == 1 ? 2 * 148 : 148;
    // up to 16 pages a row and a block for every unit: two pages a warp at most, and no second launch
    s->aligned = max_pages <= 2 * DK_WARPS && s->units <= most;
    s->n_blocks = s->aligned ? (int)s->units : (int)std::min<long long>(most, (s->units * max_pages + DK_WARPS - 1) / DK_WARPS);
    // a warp's run is counted in 31 bits
    return s->units <= 0x7fffffffll && s->units * max_pages <= 1ll << 40;
}
static size_t align256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace ag

using namespace ag;

extern "C" size_t ag_attention_decode_kv4_workspace(int B, int H_q, int H_kv, int D, int max_pages) {
    DecodeKv4Shape s;
    if (!decode_kv4_shape(B, H_q, H_kv, D, max_pages, &s)) return 0;
    return s.slots() * 8 * s.nb * D * sizeof(float) + align256(s.slots() * 8 * s.nb * sizeof(float2)) + (size_t)s.n_blocks * sizeof(int2);
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
    if (!workspace || ((uintptr_t)workspace & 15u) || workspace_bytes < need) return AG_ERR_ARG;
    ag_status st = check_arch();
    if (st != AG_OK) return st;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    DecodeKv4Args x;
    memset(&x, 0, sizeof x);
    x.Q = (const uint16_t*)Q;
    x.O = (uint16_t*)O;
    x.pages = (const uint8_t*)pool->pages;
    x.page_of = table->page_of; x.len = table->len; x.row = row;
    x.part = (float4*)workspace;
    x.stats = (float2*)((uint8_t*)workspace + s.slots() * 8 * s.nb * pool->D * sizeof(float));
    x.crossing = (int2*)((uint8_t*)x.stats + align256(s.slots() * 8 * s.nb * sizeof(float2)));
    x.B = B; x.n_pages = (int)pool->n_pages; x.H_kv = pool->H_kv; x.G = H_q / pool->H_kv;
    x.n_rows = table->n_rows; x.max_pages = table->max_pages; x.h_blocks = s.h_blocks;
    x.n_blocks = s.n_blocks; x.aligned = s.aligned;
    x.scale_log2e = 1.4426950408889634f / sqrtf((float)pool->D);
    void (*kernel)(DecodeKv4Args) = pool->D == 128 ? (s.nb == 2 ? k_attn_decode_kv4<128, 2> : k_attn_decode_kv4<128, 1>)
                                                   : (s.nb == 2 ? k_attn_decode_kv4<64, 2> : k_attn_decode_kv4<64, 1>);
    void (*join)(DecodeKv4Args) = pool->D == 128 ? (s.nb == 2 ? k_attn_join_kv4<128, 2> : k_attn_join_kv4<128, 1>)
                                                 : (s.nb == 2 ? k_attn_join_kv4<64, 2> : k_attn_join_kv4<64, 1>);
    static std::atomic<unsigned long long> attr_done{0};
    const cudaError_t attr_err = once_per_device(attr_done, [] {
        cudaError_t e = cudaFuncSetAttribute(k_attn_decode_kv4<128, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, dk_smem_bytes<128, 1>());
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k_attn_decode_kv4<128, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, dk_smem_bytes<128, 2>());
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k_attn_decode_kv4<64, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, dk_smem_bytes<64, 1>());
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k_attn_decode_kv4<64, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, dk_smem_bytes<64, 2>());
        return e;
    });
    if (attr_err != cudaSuccess) return cuda_fail(attr_err);
    // both launches may come up while the one before them on the stream finishes, and wait for it on the device
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3((unsigned)s.n_blocks);
    cfg.blockDim = dim3(DK_THREADS);
    cfg.dynamicSmemBytes = pool->D == 128 ? (s.nb == 2 ? dk_smem_bytes<128, 2>() : dk_smem_bytes<128, 1>()) : (s.nb == 2 ? dk_smem_bytes<64, 2>() : dk_smem_bytes<64, 1>());
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    AG_CUDA(cudaLaunchKernelEx(&cfg, kernel, x));
    count_launch();
    if (s.aligned) return AG_OK;
    // Side by side: 2 parts where a unit goes over few blocks (smaller blocks come up sooner: 128 requests of some 850 keys took 47.3 us with 2, 50.3 with 4 at that step),
    // 4 where there are more blocks than that (1 request of 131072 keys: 61.5 and 55.6)
    cfg.blockDim = dim3(s.nb * pool->D * 2, s.units * 4 >= s.n_blocks ? 2 : dk_join_lanes(pool->D, s.nb));
    cfg.dynamicSmemBytes = 0;
    AG_CUDA(cudaLaunchKernelEx(&cfg, join, x));
    count_launch();
    return AG_OK;
}
