// Verification of drafted tokens: which of a request's drafts stand, and the token that follows them.
//
// The walk: from a request's first token on, r = p of the token in hand; its children are tried in order.  Child x stands when u q(x) < r(x); a child that does not
// leaves r = max(r - q, 0) / sum.  Where no child is left the next token is the first v with r(0) + .. + r(v) > u_next sum(r).  (Accepting x with probability
// min(1, r(x) / q(x)) and going on with the rest of r otherwise gives x the probability r(x) whatever q is: min(q, r) + (1 - sum min(q, r)) max(r - q, 0) / sum max(r - q, 0) = r.)
//
// The rows of p and q are long (the vocabulary) and only one row of each has to be read: the one where the walk ends.  Everything before needs single entries, which all
// tokens gather at once.  A rejected child with a sibling behind it takes a pass over the row for the sum.  r itself is never stored: it follows from p, q and the sums.
// Siblings drawn without repetition: after some have been tried, q is q without those tokens, divided by left = (q's sum without them) / (q's sum).  The same passes add that up from the
// entries that are left: a q that has been used up but for little holds that little in entries which 1 minus the others (rounded, and not exactly 1 together) would lose or turn negative.
// (The sum costs 8 us of the 72 that 128 trees over 100003 take.)
// Probabilities are added up in 64 bits, in an order that no scheduling changes: a border between two tokens moves by 2^-50 of the whole.
// A cluster of blocks shares a request: each takes a stretch of the vocabulary, sums meet in distributed shared memory, and the block whose stretch holds the
// border looks for the token.  Bound: with many requests the rows' bytes, with few the chain offset -> tree -> entries -> row -> border.
// On the device: one chain of 5 over 32000 entries 9.9 us; 64 chains of 3 to 9 over 131072 (two models, 32 bits) 21 us, 3.2 TB/s, 12 of it that chain (the time over 2000 entries), 17 where the
// drafts were not drawn (one model's rows); 128 trees over 100003 without repetition 72 us, 23 of it chains, two to four passes over a row whose drafts are rejected, from the second on in the
// cache.
#include <string.h>

#include <algorithm>
#include <type_traits>

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
// The rejected children of the token in hand: r_j = max(r_{j-1} - q_j, 0) / sum_j, q_j = q / left_j without the tokens tried before.
struct Rejected {
    int n;                                 // of them
    int kept;                              // some sum was 0: r stayed as it was there
    int tried[VD_MAX];
    double inv_left[VD_MAX], inv_sum[VD_MAX];  // 1 / the share of q that is left for child j; 1 / sum_j (0: r stays; 1 for the last one: its scale does not matter)
};
// r - q / left, r normalised.  One form and one rounding for single entries and for sums over the row: where little is left of r, its entries and their sum have to agree, or what is
// normalised next is their difference.
__device__ __forceinline__ double less_q(double r, double q, double inv_left) {
    const double d = __fma_rn(-q, inv_left, r);
    return d > 0.0 ? d : 0.0;
}
// r of entry v after the first n rejected children, from p's entry and q's
template <bool DRAWN>
__device__ __noinline__ double rest_of(double p, double q, int v, const Rejected* rj, int n, bool distinct) {
    double r = p;
    bool tried = false;
#pragma unroll 1
    for (int j = 0; j < n; ++j) {
        const double is = rj->inv_sum[j], d = DRAWN ? less_q(r, tried ? 0.0 : q, rj->inv_left[j]) : rj->tried[j] == v ? 0.0 : r;
        if (is != 0.0) r = __dmul_rn(d, is);
        if (distinct && rj->tried[j] == v) tried = true;
    }
    return r;
}

struct VerifyShared {
    int parent[VD_MAX], token[VD_MAX], accepted[VD_MAX], passes[VD_MAX], more[VD_MAX];   // passes: as its parent's first child; more: siblings behind it
    float u[VD_MAX];
    double p[VD_MAX], q[VD_MAX];           // entries of the tokens in their parents' rows
    Rejected rj;
    double tried_q, left;                  // q of the tokens tried; the share of q that is left without them (0: nothing)
    double warp_sum[VD_WARPS], warp_rest[VD_WARPS], block_sum[2], block_rest[2], scan[VD_WARPS];
    int low[VD_WARPS], high[VD_WARPS];
    int hand, tried_at, state, found;
    double base;
};
__device__ __forceinline__ double value_of(float v) { return (double)v; }
__device__ __forceinline__ double value_of(uint16_t v) { return (double)__uint_as_float((uint32_t)v << 16); }
// a vector of a row as words; its entry e
template <class T, int W>
__device__ __forceinline__ uint4 load_vector(const T* at) {
    if constexpr (W == 1 && sizeof(T) == 4) return make_uint4(__float_as_uint(*at), 0, 0, 0);
    else if constexpr (W == 1) return make_uint4(*at, 0, 0, 0);
    else return *reinterpret_cast<const uint4*>(at);
}
template <class T>
__device__ __forceinline__ double from_word(const uint32_t (&w)[4], int e) {
    return (double)(sizeof(T) == 4 ? __uint_as_float(w[e % 4]) : e & 1 ? bf16_hi(w[e / 2 % 4]) : bf16_lo(w[e / 2 % 4]));
}

// A row in vectors of W entries: vector i has entries i W - lead .. i W - lead + W - 1 and, W > 1, starts on a multiple of 16 bytes in p and in q.
struct Scan {
    double sum;                            // of r over the thread's vectors
    int last, cross;                       // the last entry above 0; the first at which before + sum is above the target; -1: none
};
struct ScanRest : Scan {
    double rest;                           // of q without the tokens tried
};
// Vectors i0, i0 + step, .. below i1, of r after m rejected children; REST: also what is left of q; FIND: also the last and the first entry of Scan.  (Functions of their own: they are
// called from several places, and a call that verifies one request is bound by fetching its instructions.)
template <class T, bool DRAWN, int W, bool FIND, bool REST = false>
__device__ __noinline__ std::conditional_t<REST, ScanRest, Scan> scan_row(const T* p, const T* q, int i0, int i1, int step, int lead, int vocab, const Rejected* rj, int m, bool distinct, double before, double target) {
    constexpr int U = FIND ? 1 : W == 1 ? 4 : sizeof(T) == 4 ? 2 : 1;      // vectors in flight, of each row
    std::conditional_t<REST, ScanRest, Scan> s;
    s.sum = before;
    s.last = s.cross = -1;
    if constexpr (REST) s.rest = 0.0;
    const bool with_q = DRAWN && m > 0, kept = rj->kept != 0;
    const double il0 = with_q ? rj->inv_left[0] : 0.0;
    p -= lead;
    q -= lead;
    int near = 0;                          // REST: m where a token tried lies between the thread's vectors, and is looked for in each
    if constexpr (REST) {
#pragma unroll 1
        for (int j = 0; j < m; ++j) near = rj->tried[j] >= i0 * W - lead && rj->tried[j] < i1 * W - lead ? m : near;
    }
#pragma unroll 1
    for (int i = i0; i < i1; i += U * step) {
        uint4 pv[U], qv[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int at = i + k * step, e = at * W - lead;
            pv[k] = qv[k] = make_uint4(0, 0, 0, 0);
            if (at < i1 && e >= 0 && e + W <= vocab) {
                pv[k] = load_vector<T, W>(p + (long long)at * W);
                if (with_q) qv[k] = load_vector<T, W>(q + (long long)at * W);
            } else if (at < i1) {                              // a row's ends: entry by entry
#pragma unroll 1
                for (int x = 0; x < W; ++x) {
                    if (e + x < 0 || e + x >= vocab) continue;
                    const T a = p[(long long)at * W + x], c = with_q ? q[(long long)at * W + x] : T(0);
                    uint32_t wa, wc;
                    if constexpr (sizeof(T) == 4) wa = __float_as_uint(a), wc = __float_as_uint(c);
                    else wa = (uint32_t)a << (16 * (x & 1)), wc = (uint32_t)c << (16 * (x & 1));
                    const int word = x * (int)sizeof(T) / 4;
                    (word == 0 ? pv[k].x : word == 1 ? pv[k].y : word == 2 ? pv[k].z : pv[k].w) |= wa;
                    (word == 0 ? qv[k].x : word == 1 ? qv[k].y : word == 2 ? qv[k].z : qv[k].w) |= wc;
                }
            }
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int e0 = (i + k * step) * W - lead;
            const uint32_t pw[4] = {pv[k].x, pv[k].y, pv[k].z, pv[k].w}, qw[4] = {qv[k].x, qv[k].y, qv[k].z, qv[k].w};
            if constexpr (REST) {
                uint32_t tried = 0;
#pragma unroll 1
                for (int j = 0; j < near; ++j) {
                    const unsigned at = (unsigned)(rj->tried[j] - e0);
                    tried |= at < W ? 1u << at : 0u;
                }
                double left[W];
#pragma unroll
                for (int e = 0; e < W; ++e) left[e] = from_word<T>(qw, e);
                if (tried) {
#pragma unroll
                    for (int e = 0; e < W; ++e) left[e] = tried >> e & 1 ? 0.0 : left[e];
                }
#pragma unroll
                for (int e = 1; e < W; ++e) left[0] += left[e];
                s.rest += left[0];
            }
            double r[W];
            // (nothing beyond the ends: zeros of p stay zeros)
            if (DRAWN && !kept) {
#pragma unroll
                for (int e = 0; e < W; ++e) r[e] = less_q(from_word<T>(pw, e), from_word<T>(qw, e), il0);
#pragma unroll 1
                for (int j = 1; j < m; ++j) {
                    const double is = rj->inv_sum[j - 1], il = rj->inv_left[j];
#pragma unroll
                    for (int e = 0; e < W; ++e) r[e] = less_q(__dmul_rn(r[e], is), from_word<T>(qw, e), il);
                }
            } else {
#pragma unroll
                for (int e = 0; e < W; ++e) r[e] = from_word<T>(pw, e);
#pragma unroll 1
                for (int j = 0; j < m && !DRAWN; ++j) {
                    const double is = rj->inv_sum[j];
                    if (is == 0.0) continue;
#pragma unroll
                    for (int e = 0; e < W; ++e) r[e] = rj->tried[j] == e0 + e ? 0.0 : __dmul_rn(r[e], is);
                }
                if (DRAWN) {
#pragma unroll
                    for (int e = 0; e < W; ++e) r[e] = rest_of<DRAWN>(r[e], from_word<T>(qw, e), e0 + e, rj, m, distinct);
                }
            }
            double all = r[0];
#pragma unroll
            for (int e = 1; e < W; ++e) all += r[e];
            if (FIND) {
                double run = s.sum;
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    run += r[e];
                    if (r[e] > 0.0) {
                        s.last = e0 + e;
                        if (s.cross < 0 && run > target) s.cross = e0 + e;
                    }
                }
            }
            s.sum += all;
        }
    }
    s.sum -= before;
    return s;
}

// VEC: rows of p and of q lie alike with respect to 16 bytes
template <class T, bool DRAWN, bool VEC>
__global__ void __launch_bounds__(VD_THREADS, 2) k_verify(const VerifyArgs x) {
    constexpr int W = VEC ? 16 / (int)sizeof(T) : 1;
    __shared__ VerifyShared sh;
    dep_wait();
    dep_release();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = x.cluster > 1 ? (int)cluster_rank() : 0;
    const int seq = blockIdx.x / x.cluster;
    const bool distinct = x.distinct != 0;
    const long long first = min(max((long long)x.off[seq], 0ll), x.n_tokens), stop = min(max((long long)x.off[seq + 1], first), x.n_tokens);
    const int n = (int)min(stop - first, (long long)VD_MAX);
    const T *P = (const T*)x.P + first * x.p_stride, *Q = (const T*)x.Q + first * x.q_stride;
    if (rank == 0)
        for (long long i = first + VD_MAX + tid; i < stop; i += VD_THREADS) x.accepted[i] = 0;
    if (n == 0) {                                              // (all blocks of the cluster alike)
        if (rank == 0 && tid == 0) x.next[seq] = -1;
        return;
    }
    const float u_next = x.u_next[seq];
    if (tid < n) {
        const int parent = x.parent ? x.parent[first + tid] : tid - 1, token = x.token[first + tid];
        const bool fine = tid > 0 && parent >= 0 && parent < tid && token >= 0 && token < x.vocab;
        const float u = tid > 0 ? x.u[first + tid] : 0.f;
        const double p = fine ? value_of(P[parent * x.p_stride + token]) : 0.0, q = DRAWN && fine ? value_of(Q[parent * x.q_stride + token]) : 1.0;
        sh.parent[tid] = fine ? parent : -1;
        sh.token[tid] = token;
        sh.u[tid] = u;
        sh.accepted[tid] = tid == 0;
        sh.p[tid] = p;
        sh.q[tid] = q;
        sh.passes[tid] = fine && (double)u * q < p;
    }
    if (tid == 0) {
        sh.hand = 0;
        sh.tried_at = 1;
        sh.rj.n = sh.rj.kept = 0;
    }
    __syncthreads();
    if (tid < n) {
        int more = 0;
#pragma unroll 1
        for (int k = tid + 1; k < n; ++k) more |= sh.parent[k] == sh.parent[tid];
        sh.more[tid] = more;
    }
    int lead = 0, b0 = 0, b1 = 0, per_warp = 0, sums = 0;
    double others = 0.0;                                       // lane c: the sum of block c of the cluster
    double total;
    for (;;) {
        __syncthreads();
        // ---- the walk: every block of the cluster takes it alike, up to a rejected child with siblings behind it (state 1: the sum of what is left is wanted) or the end
        if (tid == 0) {
            int state = 0, hand = sh.hand, i = sh.tried_at;
            Rejected& rj = sh.rj;
#pragma unroll 1
            for (; i < n && !state; ++i) {
                if (sh.parent[i] != hand || (rj.n && sh.left == 0.0)) continue;        // (nothing of q is left: no draft of it)
                bool stands = sh.passes[i] != 0;
                const int t = sh.token[i];
                double left = 1.0, q = sh.q[i];
                if (rj.n) {
                    if (DRAWN && distinct) {
                        left = sh.left;
#pragma unroll 1
                        for (int j = 0; j < rj.n; ++j)
                            if (rj.tried[j] == t) q = 0.0;
                    }
                    stands = (double)sh.u[i] * (DRAWN ? q / left : 1.0) < rest_of<DRAWN>(sh.p[i], sh.q[i], t, &rj, rj.n, distinct);
                }
                if (stands) {
                    sh.accepted[i] = 1;
                    hand = i;
                    rj.n = rj.kept = 0;
                } else {
                    rj.tried[rj.n] = t;
                    rj.inv_left[rj.n] = 1.0 / left;
                    rj.inv_sum[rj.n] = 1.0;                    // (until the sum is there)
                    ++rj.n;
                    sh.left = 1.0;                             // (DISTINCT: what the sum over the row finds)
                    sh.tried_q = rj.n > 1 ? sh.tried_q + q : q;
                    state = sh.more[i];
                    if (!state) break;
                }
            }
            sh.hand = hand;
            sh.tried_at = i;
            sh.state = state;
        }
        __syncthreads();
        const int m = sh.rj.n, state = sh.state;
        // ---- the sum of r: a block has a stretch of the row's vectors, each warp a part of that
        const T *p = P + sh.hand * x.p_stride, *q = Q + sh.hand * x.q_stride;
        lead = VEC ? (int)(((uintptr_t)p & 15u) / sizeof(T)) : 0;
        const int vectors = (x.vocab + lead + W - 1) / W, per_block = (vectors + x.cluster - 1) / x.cluster;
        b0 = min(rank * per_block, vectors);
        b1 = min(b0 + per_block, vectors);
        per_warp = (b1 - b0 + VD_WARPS - 1) / VD_WARPS;
        const int w0 = min(b0 + warp * per_warp, b1), w1 = min(w0 + per_warp, b1);
        const bool with_rest = DRAWN && distinct && state == 1;
        double sum;
        if constexpr (DRAWN) {
            if (with_rest) {
                const ScanRest part = scan_row<T, DRAWN, W, false, true>(p, q, w0 + lane, w1, 32, lead, x.vocab, &sh.rj, m, distinct, 0.0, INFINITY);
                sum = part.sum;
                double rest = part.rest;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) rest += __shfl_xor_sync(0xffffffffu, rest, o);
                if (lane == 0) sh.warp_rest[warp] = rest;
            }
        }
        if (!with_rest) sum = scan_row<T, DRAWN, W, false>(p, q, w0 + lane, w1, 32, lead, x.vocab, &sh.rj, m, distinct, 0.0, INFINITY).sum;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) sh.warp_sum[warp] = sum;
        __syncthreads();
        double *block_sum = &sh.block_sum[sums & 1], *block_rest = &sh.block_rest[sums & 1];   // (two in turn: one barrier a sum)
        ++sums;
        if (warp == 0) {
            double all = lane < VD_WARPS ? sh.warp_sum[lane] : 0.0;
#pragma unroll
            for (int o = VD_WARPS / 2; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
            if (lane == 0) *block_sum = all;
        } else if (with_rest && warp == 1) {
            double all = lane < VD_WARPS ? sh.warp_rest[lane] : 0.0;
#pragma unroll
            for (int o = VD_WARPS / 2; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
            if (lane == 0) *block_rest = all;
        }
        if (x.cluster > 1) cluster_arrive_wait();
        else __syncthreads();
        others = lane >= x.cluster ? 0.0 : x.cluster > 1 ? peer_double(block_sum, lane) : *block_sum;
        total = others;
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        total = __shfl_sync(0xffffffffu, total, 0);
        if (with_rest && warp == 0) {
            double left = lane >= x.cluster ? 0.0 : x.cluster > 1 ? peer_double(block_rest, lane) : *block_rest;
#pragma unroll
            for (int o = 4; o > 0; o >>= 1) left += __shfl_xor_sync(0xffffffffu, left, o);
            if (lane == 0) sh.left = left > 0.0 ? left / (left + sh.tried_q) : 0.0;
        }
        if (state == 1) {
            if (tid == 0) {
                sh.rj.inv_sum[m - 1] = total > 0.0 ? 1.0 / total : 0.0;
                sh.rj.kept |= !(total > 0.0);
            }
        } else if (total == 0.0 && m > 0 && sh.rj.inv_sum[m - 1] != 0.0) {
            // nothing is left above q: r stays (nobody is left to be tried: the walk ends at once)
            __syncthreads();
            if (tid == 0) {
                sh.rj.inv_sum[m - 1] = 0.0;
                sh.rj.kept = 1;
                sh.tried_at = n;
            }
        } else {
            break;
        }
    }

    // ---- the token that follows: the block, then the warp's part, then the entry that holds the border - the first whose running sum is above it, or the last with any weight
    const double target = (double)u_next * total;
    if (rank == 0 && tid < n) x.accepted[first + tid] = sh.accepted[tid];
    if (warp == 0) {
        // among `count` sums, lane by lane: the first that takes the running sum above the target, else the last above 0; the running sum in front of it
        auto choose = [&](double v, double from, double& before) -> int {
            double inc = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double up = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += up;
            }
            const unsigned some = __ballot_sync(0xffffffffu, v > 0.0), above = __ballot_sync(0xffffffffu, v > 0.0 && from + inc > target);
            const int at = above ? __ffs(above) - 1 : some ? 31 - __clz(some) : -1;
            before = from + __shfl_sync(0xffffffffu, inc - v, max(at, 0));
            return at;
        };
        double before, base;
        const int block = choose(others, 0.0, before);
        int found = -1;
        if (block == rank) found = choose(lane < VD_WARPS ? sh.warp_sum[lane] : 0.0, before, base);
        if (lane == 0) {
            sh.found = found;
            if (found >= 0) sh.base = base;
            if (block < 0 && rank == 0) x.next[seq] = -1;
        }
    }
    __syncthreads();
    if (sh.found >= 0) {
        // thread t looks at a run of the found warp's vectors; then the one whose run holds the border looks for the entry
        const int m = sh.rj.n;
        const T *p = P + sh.hand * x.p_stride, *q = Q + sh.hand * x.q_stride;
        const int s0 = min(b0 + sh.found * per_warp, b1), s1 = min(s0 + per_warp, b1), run = (s1 - s0 + VD_THREADS - 1) / VD_THREADS;
        const int t0 = min(s0 + tid * run, s1), t1 = min(t0 + run, s1);
        double before = 0.0;
        Scan s{0.0, -1, -1};
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {
            if (pass == 0 || (s.sum > 0.0 && before + s.sum > target)) s = scan_row<T, DRAWN, W, true>(p, q, t0, t1, 1, lead, x.vocab, &sh.rj, m, distinct, before, pass ? target : INFINITY);
            if (pass) break;
            double inc = s.sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double up = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += up;
            }
            if (lane == 31) sh.scan[warp] = inc;
            __syncthreads();
            before = lane < warp ? sh.scan[lane % VD_WARPS] : 0.0;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
            before += sh.base + inc - s.sum;
        }
        const int cross = __reduce_min_sync(0xffffffffu, s.cross < 0 ? x.vocab : s.cross), last = __reduce_max_sync(0xffffffffu, s.last);
        if (lane == 0) {
            sh.low[warp] = cross;
            sh.high[warp] = last;
        }
        __syncthreads();
        if (warp == 0) {
            const int low = __reduce_min_sync(0xffffffffu, sh.low[lane % VD_WARPS]), high = __reduce_max_sync(0xffffffffu, sh.high[lane % VD_WARPS]);
            if (lane == 0) x.next[seq] = low < x.vocab ? low : high;
        }
    }
    if (x.cluster > 1) cluster_arrive_wait();                  // nobody leaves while its sum may still be read
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
    if (!v->off || !v->u_next || !v->next) return AG_ERR_ARG;
    if (v->n_tokens > 0 ? !v->new_off != !v->from : v->from && !v->new_off) return AG_ERR_ARG;       // (an array of no tokens may be NULL)
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
    // both models' rows alike with respect to 16 bytes
    const int64_t size = v->type == AG_F32 ? 4 : 2;
    const bool vec = !v->Q || (((uintptr_t)v->P - (uintptr_t)v->Q) % 16 == 0 && (v->p_stride - v->q_stride) * size % 16 == 0);
    auto pick = [&](auto type) {
        using T = decltype(type);
        return v->Q ? (vec ? k_verify<T, true, true> : k_verify<T, true, false>) : k_verify<T, false, true>;
    };
    void (*kernel)(VerifyArgs) = v->type == AG_F32 ? pick(0.f) : pick((uint16_t)0);
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
