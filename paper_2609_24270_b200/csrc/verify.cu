// Verification of drafted tokens: which of a request's drafts stand, and the token that follows them.
//
// The walk: from a request's first token on, r = p of the token in hand; its children are tried in order.  Child x stands when u q(x) < r(x); a child that does not
// leaves r = max(r - q, 0) / sum.  Where no child is left the next token is the first v with r(0) + .. + r(v) > u_next sum(r).  (Accepting x with probability
// min(1, r(x) / q(x)) and going on with the rest of r otherwise gives x the probability r(x) whatever q is: min(q, r) + (1 - sum min(q, r)) max(r - q, 0) / sum max(r - q, 0) = r.)
//
// The rows of p and q are long (the vocabulary) and only one row of each has to be read: the one where the walk ends.  Everything before needs single entries, which all
// tokens gather at once.  A rejected child with a sibling behind it takes a pass over the row for the sum.  r itself is never stored: it follows from p, q and the sums.
// Probabilities are added up in 64 bits, in an order that no scheduling changes: a border between two tokens moves by 2^-50 of the whole.
// A cluster of blocks shares a request: each takes a stretch of the vocabulary, sums meet in distributed shared memory, and the block whose stretch holds the
// border looks for the token.  Bound: with many requests the rows' bytes, with few the chain offset -> tree -> entries -> row -> border.
#include <string.h>

#include <algorithm>

#include "kv4.cuh"

namespace ag {

constexpr int VD_THREADS = 512;
constexpr int VD_WARPS = VD_THREADS / 32;
constexpr int VD_MAX = AG_TREE_MAX;

struct VerifyArgs {
    const void *P, *Q;
    long long p_stride, q_stride;
    const int32_t *off, *parent, *token;
    const float *u, *u_next;
    int32_t *accepted, *next;
    int vocab, distinct, n_seq, cluster;
    long long n_tokens;
};

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive_wait() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ double peer_double(const double* own, uint32_t rank) {   // the same variable in another block of the cluster
    uint32_t a;
    double v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(own)), "r"(rank));
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(a) : "memory");
    return v;
}
template <class T>
__device__ __forceinline__ double entry(const T* row, long long v);
template <>
__device__ __forceinline__ double entry<float>(const float* row, long long v) { return (double)row[v]; }
template <>
__device__ __forceinline__ double entry<uint16_t>(const uint16_t* row, long long v) { return (double)__uint_as_float((uint32_t)row[v] << 16); }

// The rejected children of the token in hand: r_j = max(r_{j-1} - q_j, 0) / sum_j, q_j = q / left_j without the tokens tried before.
struct Rejected {
    int n;                                 // of them
    int tried[VD_MAX];
    double left[VD_MAX], inv_sum[VD_MAX];  // what is left of q's 1 for child j; 1 / sum_j (0: r stays as it is; 1 for the last one: its scale does not matter)
};

// r of entry v after the first `n` rejected children; q: its q entry (drawn) or nothing (not drawn)
template <bool DRAWN>
__device__ __forceinline__ double rest_of(double p, double q, int v, const Rejected& rj, int n, bool distinct) {
    double r = p;
    bool tried = false;
    for (int j = 0; j < n; ++j) {
        if (DRAWN) {
            const double d = fmax(r - (tried ? 0.0 : q / rj.left[j]), 0.0);
            if (rj.inv_sum[j] != 0.0) r = d * rj.inv_sum[j];
            if (distinct && rj.tried[j] == v) tried = true;
        } else {
            if (rj.inv_sum[j] != 0.0) r = rj.tried[j] == v ? 0.0 : r * rj.inv_sum[j];
        }
    }
    return r;
}

struct VerifyShared {
    int parent[VD_MAX], token[VD_MAX], accepted[VD_MAX];
    float u[VD_MAX];
    double p[VD_MAX], q[VD_MAX];           // entries of the tokens in their parents' rows
    Rejected rj;
    double warp_sum[VD_WARPS], block_sum, scan[VD_WARPS];
    int hand, tried_at, state, found;
    double base;
};

template <class T, bool DRAWN>
__global__ void __launch_bounds__(VD_THREADS) k_verify(const VerifyArgs x) {
    __shared__ VerifyShared sh;
    dep_wait();
    dep_release();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = x.cluster > 1 ? (int)cluster_rank() : 0;
    const int seq = blockIdx.x / x.cluster;
    const long long first = min(max((long long)x.off[seq], 0ll), x.n_tokens), stop = min(max((long long)x.off[seq + 1], first), x.n_tokens);
    const int n = (int)min(stop - first, (long long)VD_MAX);
    const T *P = (const T*)x.P + first * x.p_stride, *Q = (const T*)x.Q + first * x.q_stride;
    if (rank == 0)
        for (long long i = first + VD_MAX + tid; i < stop; i += VD_THREADS) x.accepted[i] = 0;
    if (n == 0) {                                              // (all blocks of the cluster alike)
        if (rank == 0 && tid == 0) x.next[seq] = -1;
        return;
    }
    if (tid < n) {
        const int parent = x.parent ? x.parent[first + tid] : tid - 1, token = x.token[first + tid];
        const bool fine = tid > 0 && parent >= 0 && parent < tid && token >= 0 && token < x.vocab;
        sh.parent[tid] = fine ? parent : -1;
        sh.token[tid] = token;
        sh.u[tid] = tid > 0 ? x.u[first + tid] : 0.f;
        sh.accepted[tid] = tid == 0;
        sh.p[tid] = fine ? entry(P + parent * x.p_stride, token) : 0.0;
        sh.q[tid] = DRAWN && fine ? entry(Q + parent * x.q_stride, token) : 1.0;
    }
    if (tid == 0) {
        sh.hand = 0;
        sh.tried_at = 1;
        sh.rj.n = 0;
    }
    // this block's stretch of the vocabulary, and the warp's of it
    const int per_block = (x.vocab + x.cluster - 1) / x.cluster, b0 = min(rank * per_block, x.vocab), b1 = min(b0 + per_block, x.vocab);
    const int per_warp = ((b1 - b0 + VD_WARPS - 1) / VD_WARPS + 31) / 32 * 32, w0 = min(b0 + warp * per_warp, b1), w1 = min(w0 + per_warp, b1);

    // sum of r after m rejected children (the last of them not divided yet) over the warp's stretch; all blocks' sum in return
    auto row_sum = [&](int m) -> double {
        const T *p = P + sh.hand * x.p_stride, *q = Q + sh.hand * x.q_stride;
        double sum = 0.0;
        for (int v = w0 + lane; v < w1; v += 32) sum += rest_of<DRAWN>(entry(p, v), DRAWN && m > 0 ? entry(q, v) : 0.0, v, sh.rj, m, x.distinct != 0);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        __syncthreads();
        if (lane == 0) sh.warp_sum[warp] = sum;
        __syncthreads();
        if (tid == 0) {
            double all = 0.0;
            for (int w = 0; w < VD_WARPS; ++w) all += sh.warp_sum[w];
            sh.block_sum = all;
        }
        if (x.cluster == 1) {
            __syncthreads();
            return sh.block_sum;
        }
        cluster_arrive_wait();
        double all = 0.0;
        for (int c = 0; c < x.cluster; ++c) all += peer_double(&sh.block_sum, c);
        cluster_arrive_wait();                                 // (block_sum has been read by everybody)
        return all;
    };

    // ---- the walk: every block of the cluster takes it alike
    for (;;) {
        __syncthreads();
        if (tid == 0) {
            int state = 0;                                     // 1: a sum is wanted
            for (int i = sh.tried_at; i < n && !state; ++i) {
                if (sh.parent[i] != sh.hand) continue;
                Rejected& rj = sh.rj;
                const int t = sh.token[i];
                const double r = rest_of<DRAWN>(sh.p[i], sh.q[i], t, rj, rj.n, x.distinct != 0);
                double left = 1.0, q = sh.q[i];
                if (DRAWN && x.distinct) {
                    if (rj.n) {
                        // what the child before left, without that child itself
                        left = rj.left[rj.n - 1];
                        bool again = false;
                        for (int j = 0; j + 1 < rj.n; ++j) again |= rj.tried[j] == rj.tried[rj.n - 1];
                        for (int k = 1; k < n && !again; ++k)
                            if (sh.parent[k] == sh.hand && sh.token[k] == rj.tried[rj.n - 1]) {
                                left -= sh.q[k];
                                again = true;
                            }
                    }
                    for (int j = 0; j < rj.n; ++j)
                        if (rj.tried[j] == t) q = 0.0;
                }
                if ((double)sh.u[i] * (DRAWN ? q / left : 1.0) < r) {
                    sh.accepted[i] = 1;
                    sh.hand = i;
                    rj.n = 0;
                } else {
                    rj.tried[rj.n] = t;
                    rj.left[rj.n] = left;
                    rj.inv_sum[rj.n] = 1.0;                    // (until the sum is there)
                    ++rj.n;
                    sh.tried_at = i + 1;
                    for (int k = i + 1; k < n; ++k)
                        if (sh.parent[k] == sh.hand) state = 1;
                }
            }
            sh.state = state;
        }
        __syncthreads();
        if (sh.state == 0) break;
        const double sum = row_sum(sh.rj.n);
        if (tid == 0) sh.rj.inv_sum[sh.rj.n - 1] = sum > 0.0 ? 1.0 / sum : 0.0;
    }

    // ---- the token that follows
    const int m = sh.rj.n;
    double total = row_sum(m);
    if (total == 0.0 && m > 0 && sh.rj.inv_sum[m - 1] != 0.0) {    // nothing is left above q (the two are equal but for roundings): r stays
        __syncthreads();
        if (tid == 0) sh.rj.inv_sum[m - 1] = 0.0;
        __syncthreads();
        total = row_sum(m);
    }
    const double target = (double)x.u_next[seq] * total;
    if (rank == 0 && tid < n) x.accepted[first + tid] = sh.accepted[tid];
    // the block, then the warp's stretch, then the entry that holds the border: the first whose running sum is above it, or the last with any weight
    if (tid == 0) {
        double before = 0.0, at = 0.0;
        int mine = -1, last = -1;
        double last_before = 0.0;
        for (int c = 0; c < x.cluster; ++c) {
            const double s = x.cluster == 1 ? sh.block_sum : peer_double(&sh.block_sum, c);
            if (mine < 0 && s > 0.0) {
                last = c;
                last_before = before;
                if (before + s > target) {
                    mine = c;
                    at = before;
                }
            }
            before += s;
        }
        if (mine < 0) {
            mine = last;
            at = last_before;
        }
        sh.found = -1;
        if (mine == rank) {
            int w_last = -1;
            double w_before = at, l_before = at;
            sh.found = -2;
            for (int w = 0; w < VD_WARPS; ++w) {
                if (sh.warp_sum[w] > 0.0) {
                    w_last = w;
                    l_before = w_before;
                    if (w_before + sh.warp_sum[w] > target) break;
                }
                w_before += sh.warp_sum[w];
            }
            sh.found = w_last;
            sh.base = l_before;
        } else if (mine < 0 && rank == 0) {
            x.next[seq] = -1;
        }
    }
    if (x.cluster > 1) cluster_arrive_wait();                  // nobody leaves while its sum is still read
    else __syncthreads();
    if (sh.found < 0) return;
    // thread t looks at a run of the found warp's stretch
    const int s0 = min(b0 + sh.found * per_warp, b1), s1 = min(s0 + per_warp, b1), run = (s1 - s0 + VD_THREADS - 1) / VD_THREADS;
    const int t0 = min(s0 + tid * run, s1), t1 = min(t0 + run, s1);
    const T *p = P + sh.hand * x.p_stride, *q = Q + sh.hand * x.q_stride;
    auto weight = [&](int v) { return rest_of<DRAWN>(entry(p, v), DRAWN && m > 0 ? entry(q, v) : 0.0, v, sh.rj, m, x.distinct != 0); };
    double sum = 0.0;
    int last = -1;
    for (int v = t0; v < t1; ++v) {
        const double w = weight(v);
        if (w > 0.0) last = v;
        sum += w;
    }
    double inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double up = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += up;
    }
    if (lane == 31) sh.scan[warp] = inc;
    __syncthreads();
    double before = sh.base + inc - sum;
    for (int w = 0; w < warp; ++w) before += sh.scan[w];
    // the first thread whose run crosses the border, or the last one with weight
    int cross = x.vocab, any = -1;
    if (last >= 0) {
        any = last;
        double at = before;
        for (int v = t0; v < t1; ++v) {
            const double w = weight(v);
            at += w;
            if (w > 0.0 && at > target) {
                cross = v;
                break;
            }
        }
    }
    cross = __reduce_min_sync(0xffffffffu, cross);
    any = __reduce_max_sync(0xffffffffu, any);
    __syncthreads();
    int* lows = reinterpret_cast<int*>(sh.warp_sum);
    if (lane == 0) {
        lows[2 * warp] = cross;
        lows[2 * warp + 1] = any;
    }
    __syncthreads();
    if (tid == 0) {
        for (int w = 0; w < VD_WARPS; ++w) {
            cross = min(cross, lows[2 * w]);
            any = max(any, lows[2 * w + 1]);
        }
        x.next[seq] = cross < x.vocab ? cross : any;
    }
}

// new_off[s] = accepted tokens in front of request s, from[j] = the j-th accepted token: one block, thread by thread over the tokens
__global__ void __launch_bounds__(1024) k_verify_pack(const int32_t* accepted, const int32_t* off, int n_seq, int n_tokens, int32_t* new_off, int32_t* from) {
    __shared__ int warp_sum[32];
    dep_wait();
    dep_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int base = 0;
    const int lo = off[0], hi = off[n_seq];                    // (tokens of no request)
    for (int t0 = 0; t0 < n_tokens; t0 += 1024) {
        const int i = t0 + threadIdx.x;
        const int a = i < n_tokens && i >= lo && i < hi ? accepted[i] : 0;
        const unsigned set = __ballot_sync(0xffffffffu, a != 0);
        if (lane == 0) warp_sum[warp] = __popc(set);
        __syncthreads();
        const int mine = warp_sum[lane];
        int inc = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += up;
        }
        const int before = base + __shfl_sync(0xffffffffu, inc - mine, warp) + __popc(set & ((1u << lane) - 1u));
        base += __shfl_sync(0xffffffffu, inc, 31);
        if (a) from[before] = i;
        __syncthreads();
    }
    for (int j = base + threadIdx.x; j < n_tokens; j += 1024) from[j] = -1;
    __syncthreads();                                           // from is complete, and visible to the block
    // accepted tokens in front of off[s]: the first j with from[j] >= off[s]
    for (int s = threadIdx.x; s <= n_seq; s += 1024) {
        const int o = off[s];
        int a = 0, b = base;
        while (a < b) {
            const int mid = (a + b) >> 1;
            if (from[mid] < o) a = mid + 1; else b = mid;
        }
        new_off[s] = a;
    }
}

}  // namespace ag

using namespace ag;

extern "C" ag_status ag_verify_drafts(const ag_draft_verification* v, void* cuda_stream) {
    if (!v || v->n_seq < 0 || v->n_tokens < 0 || v->n_tokens >= (1ll << 30)) return AG_ERR_ARG;
    if (v->n_seq == 0) return AG_OK;
    if ((v->type != AG_F32 && v->type != AG_BF16) || v->vocab < 1 || v->vocab > (1 << 24) || v->p_stride < v->vocab || (v->Q && v->q_stride < v->vocab)) return AG_ERR_ARG;
    if (!v->off || !v->u_next || !v->next || !v->new_off != !v->from) return AG_ERR_ARG;
    if (v->n_tokens > 0 && (!v->P || !v->token || !v->u || !v->accepted)) return AG_ERR_ARG;
    const uintptr_t word = (uintptr_t)v->off | (uintptr_t)v->parent | (uintptr_t)v->token | (uintptr_t)v->u | (uintptr_t)v->u_next | (uintptr_t)v->accepted |
                           (uintptr_t)v->next | (uintptr_t)v->new_off | (uintptr_t)v->from;
    if ((word & 3u) || (((uintptr_t)v->P | (uintptr_t)v->Q) & (v->type == AG_F32 ? 3u : 1u))) return AG_ERR_ARG;
    ag_status st = check_arch();
    if (st != AG_OK) return st;
    VerifyArgs x;
    memset(&x, 0, sizeof x);
    x.P = v->P; x.Q = v->Q; x.p_stride = v->p_stride; x.q_stride = v->q_stride;
    x.off = v->off; x.parent = v->parent; x.token = v->token; x.u = v->u; x.u_next = v->u_next;
    x.accepted = v->accepted; x.next = v->next;
    x.vocab = v->vocab; x.distinct = v->distinct; x.n_seq = v->n_seq; x.n_tokens = v->n_tokens;
    // as many blocks to a request as the chip has room for, two blocks an SM
    x.cluster = 8;
    while (x.cluster > 1 && (long long)v->n_seq * x.cluster > 2 * 148) x.cluster /= 2;
    if ((long long)v->n_seq * x.cluster > 0x7fffffffll) return AG_ERR_ARG;
    void (*kernel)(VerifyArgs) = v->type == AG_F32 ? (v->Q ? k_verify<float, true> : k_verify<float, false>) : (v->Q ? k_verify<uint16_t, true> : k_verify<uint16_t, false>);
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3((unsigned)(v->n_seq * x.cluster));
    cfg.blockDim = dim3(VD_THREADS);
    cfg.stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)x.cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    AG_CUDA(cudaLaunchKernelEx(&cfg, kernel, x));
    count_launch();
    if (v->new_off) {
        AG_CUDA(launch_dependent(k_verify_pack, 1, 1024, cfg.stream, (const int32_t*)v->accepted, v->off, v->n_seq, (int)v->n_tokens, v->new_off, v->from));
        count_launch();
    }
    return AG_OK;
}
