// Attention of drafted tokens over the 4-bit cache and over one another (a tree): see include/asymgemm.h, "drafted tokens".
#include <math.h>
#include <string.h>

#include <algorithm>

#include "kv4.cuh"

namespace ag {

constexpr int TA_THREADS = 256;
constexpr int TA_ROWS = 4;                 // rows (token, head of the group) of a warp

struct TreeArgs {
    const uint16_t *Q, *K, *V;
    uint16_t* O;
    const uint8_t* pages;
    long long q_stride, k_stride, v_stride, o_stride, n_tokens;
    const int32_t *row, *off, *parent, *page_of, *len;
    int H_q, H_kv, G, n_seq, n_rows, max_pages, n_pages, max_tokens, tiles;
    float scale_log2e;
};

template <int D>
__global__ void __launch_bounds__(TA_THREADS) k_tree(const TreeArgs x) {
    constexpr int WARPS = TA_THREADS / 32, BLOCK_ROWS = WARPS * TA_ROWS;
    extern __shared__ float tree_smem[];
    float* ks = tree_smem;                                     // [64][D + 1]
    float* vs = ks + 64 * (D + 1);                             // [64][D]
    float* qs = vs + 64 * D;                                   // [BLOCK_ROWS][D]
    __shared__ unsigned long long sees[AG_TREE_MAX];
    __shared__ float ps[WARPS][64];
    dep_wait();
    dep_release();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int tile = blockIdx.x % x.tiles, hk = blockIdx.x / x.tiles % x.H_kv, seq = blockIdx.x / x.tiles / x.H_kv;
    const long long first = min(max((long long)x.off[seq], 0ll), x.n_tokens), stop = min(max((long long)x.off[seq + 1], first), x.n_tokens);
    const int n = (int)min(stop - first, (long long)x.max_tokens);
    if (tile == 0)
        for (long long i = first + n; i < stop; ++i)
            for (int d = tid; d < x.G * D; d += TA_THREADS) x.O[i * x.o_stride + (long long)hk * x.G * D + d] = 0;
    const int rows = n * x.G, r0 = tile * BLOCK_ROWS;
    if (r0 >= rows) return;
    const int table_row = x.row ? x.row[seq] : seq;
    const int len = table_row >= 0 && table_row < x.n_rows ? (int)min((long long)max(x.len[table_row], 0), 64ll * x.max_pages) : 0;
    if (tid < n) {
        unsigned long long m = 0;
        for (int i = tid; i >= 0;) {
            m |= 1ull << i;
            const int p = x.parent ? x.parent[first + i] : i - 1;
            i = p < i ? p : -1;
        }
        sees[tid] = m;
    }
    for (int i = tid; i < BLOCK_ROWS * D; i += TA_THREADS) {
        const int r = r0 + i / D;
        qs[i] = r < rows ? __uint_as_float((uint32_t)x.Q[(first + r / x.G) * x.q_stride + (hk * x.G + r % x.G) * D + i % D] << 16) * x.scale_log2e : 0.f;
    }
    float m[TA_ROWS], l[TA_ROWS], o[TA_ROWS][D / 32];
#pragma unroll
    for (int i = 0; i < TA_ROWS; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int d = 0; d < D / 32; ++d) o[i][d] = 0.f;
    }
    const int pages = (len + 63) / 64;
#pragma unroll 1
    for (int c = 0; c <= pages; ++c) {                         // the pages, then the drafted tokens
        __syncthreads();
        unsigned long long there = ~0ull;
        if (c < pages) {
            const int page = x.page_of[(size_t)table_row * x.max_pages + c];
            if (page < 0 || page >= x.n_pages) continue;
            if (len - c * 64 < 64) there = (1ull << (len - c * 64)) - 1;
            const uint8_t* block = x.pages + ((size_t)page * x.H_kv + hk) * kv4_head_bytes(D);
            for (int i = tid; i < 2 * 64 * D; i += TA_THREADS) {
                const int which = i / (64 * D), tok = i / D % 64, d = i % D;
                int at, high;
                if (which == 0) {
                    at = kv4_k_word<D>(tok, d / 32, d % 32 / 8) + d % 8 / 2;
                    high = d & 1;
                } else {
                    at = kv4_v_word<D>(tok, d % 16 / 8, d % 8) + d / 32;
                    high = d / 16 & 1;
                }
                const uint32_t pair = *reinterpret_cast<const uint32_t*>(block + kv4_scale_word<D>(which, tok, d / 32));
                const float v = __bfloat162float(__float2bfloat16_rn(fmaf((float)(block[at] >> (4 * high) & 15), bf16_lo(pair), bf16_hi(pair))));
                (which ? vs + tok * D : ks + tok * (D + 1))[d] = v;
            }
        } else {
            there = n < 64 ? (1ull << n) - 1 : ~0ull;
            for (int i = tid; i < 2 * n * D; i += TA_THREADS) {
                const int which = i / (n * D), tok = i / D % n, d = i % D;
                const uint16_t* from = which ? x.V + (first + tok) * x.v_stride : x.K + (first + tok) * x.k_stride;
                (which ? vs + tok * D : ks + tok * (D + 1))[d] = __uint_as_float((uint32_t)from[hk * D + d] << 16);
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TA_ROWS; ++i) {
            const int r = r0 + warp * TA_ROWS + i;
            if (r >= rows) break;
            const unsigned long long seen = c < pages ? there : there & sees[r / x.G];
            const float* q = qs + (warp * TA_ROWS + i) * D;
            float s0 = 0.f, s1 = 0.f;
            for (int d = 0; d < D; ++d) {
                s0 = fmaf(q[d], ks[lane * (D + 1) + d], s0);
                s1 = fmaf(q[d], ks[(lane + 32) * (D + 1) + d], s1);
            }
            if (!(seen >> lane & 1)) s0 = -INFINITY;
            if (!(seen >> (lane + 32) & 1)) s1 = -INFINITY;
            float top = fmaxf(s0, s1);
            for (int w = 1; w < 32; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
            const float now = fmaxf(m[i], top), ref = now == -INFINITY ? 0.f : now;
            const float f = m[i] == -INFINITY ? 0.f : ex2_ftz(m[i] - ref);
            m[i] = now;
            const float p0 = ex2_ftz(s0 - ref), p1 = ex2_ftz(s1 - ref);
            float sum = p0 + p1;
            for (int w = 1; w < 32; w <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
            l[i] = l[i] * f + sum;
#pragma unroll
            for (int d = 0; d < D / 32; ++d) o[i][d] *= f;
            __syncwarp();
            ps[warp][lane] = p0;
            ps[warp][lane + 32] = p1;
            __syncwarp();
#pragma unroll 1
            for (int j = 0; j < 64; ++j) {
                const float p = ps[warp][j];
                if (!(seen >> j & 1)) continue;
#pragma unroll
                for (int d = 0; d < D / 32; ++d) o[i][d] = fmaf(p, vs[j * D + d * 32 + lane], o[i][d]);
            }
        }
    }
    for (int i = 0; i < TA_ROWS; ++i) {
        const int r = r0 + warp * TA_ROWS + i;
        if (r >= rows) break;
        const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
        uint16_t* out = x.O + (first + r / x.G) * x.o_stride + (hk * x.G + r % x.G) * D;
#pragma unroll
        for (int d = 0; d < D / 32; ++d) out[d * 32 + lane] = __bfloat16_as_ushort(__float2bfloat16_rn(o[i][d] * inv));
    }
}

static bool tree_shape_ok(long long n_seq, int max_tokens, int H_q, int H_kv, int D, int max_pages) {
    return n_seq >= 1 && max_tokens >= 1 && max_tokens <= AG_TREE_MAX && H_kv >= 1 && H_kv <= 1024 && H_q >= H_kv && H_q % H_kv == 0 && H_q / H_kv <= 64 &&
           (D == 64 || D == 128) && max_pages >= 1 && max_pages < (1 << 25);
}

}  // namespace ag

using namespace ag;

extern "C" size_t ag_attention_tree_kv4_workspace(int n_seq, int max_tokens, int H_q, int H_kv, int D, int max_pages) {
    return tree_shape_ok(n_seq, max_tokens, H_q, H_kv, D, max_pages) ? 16 : 0;
}

extern "C" ag_status attention_tree_kv4(const ag_tree_attention* a, const ag_kv4_pool* pool, const ag_kv4_table* table, void* workspace, size_t workspace_bytes,
                                        void* cuda_stream) {
    if (!a || !kv4_pool_ok(pool) || !kv4_table_ok(table) || a->n_seq < 0 || a->n_tokens < 0 || a->n_tokens >= (1ll << 30)) return AG_ERR_ARG;
    if (a->n_seq == 0 || a->n_tokens == 0) return AG_OK;
    const int D = pool->D, H_kv = pool->H_kv;
    if (!tree_shape_ok(a->n_seq, a->max_tokens, a->H_q, H_kv, D, table->max_pages) || !a->Q || !a->K || !a->V || !a->O || !a->off || !(a->scale >= 0.f) || a->scale > 3.4e38f ||
        (!a->row && a->n_seq > table->n_rows))
        return AG_ERR_ARG;
    if ((((uintptr_t)a->Q | (uintptr_t)a->K | (uintptr_t)a->V | (uintptr_t)a->O) & 15u) || (((uintptr_t)a->row | (uintptr_t)a->off | (uintptr_t)a->parent) & 3u))
        return AG_ERR_ARG;
    const int64_t wq = (int64_t)a->H_q * D, wk = (int64_t)H_kv * D;
    if (a->q_stride < wq || a->o_stride < wq || a->k_stride < wk || a->v_stride < wk || ((a->q_stride | a->k_stride | a->v_stride | a->o_stride) % 8)) return AG_ERR_ARG;
    if (!workspace || ((uintptr_t)workspace & 15u) || workspace_bytes < ag_attention_tree_kv4_workspace(a->n_seq, a->max_tokens, a->H_q, H_kv, D, table->max_pages))
        return AG_ERR_ARG;
    ag_status st = check_arch();
    if (st != AG_OK) return st;
    TreeArgs x;
    memset(&x, 0, sizeof x);
    x.Q = (const uint16_t*)a->Q; x.K = (const uint16_t*)a->K; x.V = (const uint16_t*)a->V; x.O = (uint16_t*)a->O;
    x.pages = (const uint8_t*)pool->pages;
    x.q_stride = a->q_stride; x.k_stride = a->k_stride; x.v_stride = a->v_stride; x.o_stride = a->o_stride; x.n_tokens = a->n_tokens;
    x.row = a->row; x.off = a->off; x.parent = a->parent; x.page_of = table->page_of; x.len = table->len;
    x.H_q = a->H_q; x.H_kv = H_kv; x.G = a->H_q / H_kv; x.n_seq = a->n_seq; x.n_rows = table->n_rows; x.max_pages = table->max_pages; x.n_pages = (int)pool->n_pages;
    x.max_tokens = a->max_tokens;
    x.tiles = (a->max_tokens * x.G + TA_THREADS / 32 * TA_ROWS - 1) / (TA_THREADS / 32 * TA_ROWS);
    x.scale_log2e = 1.4426950408889634f * (a->scale > 0.f ? a->scale : 1.f / sqrtf((float)D));
    const long long blocks = (long long)x.tiles * H_kv * a->n_seq;
    if (blocks > 0x7fffffffll) return AG_ERR_ARG;
    const int smem = (64 * (2 * D + 1) + TA_THREADS / 32 * TA_ROWS * D) * (int)sizeof(float);
    static std::atomic<unsigned long long> attr_done{0};
    const cudaError_t attr_err = once_per_device(attr_done, [] {
        cudaError_t e = cudaFuncSetAttribute(k_tree<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, 128 * 1024);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k_tree<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, 128 * 1024);
        return e;
    });
    if (attr_err != cudaSuccess) return cuda_fail(attr_err);
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    if (D == 128) k_tree<128><<<(unsigned)blocks, TA_THREADS, smem, stream>>>(x);
    else k_tree<64><<<(unsigned)blocks, TA_THREADS, smem, stream>>>(x);
    AG_CUDA(cudaGetLastError());
    count_launch();
    return AG_OK;
}
