// The paged 4-bit key/value cache: quantising new tokens into pages, reading them back, and the device-side page tables
// (growing rows, forking, freeing, compacting).  Nothing here waits on the host or spins on the device; every call may be captured
// into a graph.  All page bookkeeping is in integers and does not depend on the order of blocks or atomics.
#include <string.h>

#include <algorithm>

#include "kv4.cuh"

namespace ag {

// ---- store and load ---------------------------------------------------------------------------------------------------
// D / 16 lanes hold a row, sixteen elements each: a lane's K codes are two words of the page, the V codes are transposed across lanes
// (kv4_transpose) so that a lane writes whole words of the fragment order as well.  With eight elements a lane the part of the work that goes by
// lanes (addresses, scales, exchanges) took twice as long: 86 and 51 us for 46k tokens x 8 heads stored and read back,
// now 60 and 42; the store is bound by instructions still (82 % of the issue slots), the load by its scattered eight-byte pieces of V.
//
// A block takes U times 128 / L neighbouring tokens of one head: the words of neighbouring V rows share sectors, and U rows a lane are in
// flight together (a row's chain slot -> page -> row is some 2 us long).
constexpr int KS_THREADS = 256;
constexpr int KS_ROWS = 2;                           // U of large calls; small ones take 1, for more blocks

template <int D, int U>
__global__ void __launch_bounds__(KS_THREADS) k_kv4_store(uint8_t* pages, long long n_slots, int H_kv, const uint16_t* K,
                                                          const uint16_t* V, long long n_tokens, long long k_stride, long long v_stride,
                                                          const int32_t* slot) {
    dep_wait();
    dep_release();
    constexpr int L = D / 16, TOK = KS_THREADS / 2 / L;             // lanes of a row, tokens of the block side by side
    const int l = threadIdx.x % L, which = threadIdx.x / 32 & 1;    // a warp has rows of K or rows of V
    const int head = blockIdx.x % H_kv;
    const long long tok0 = (long long)(blockIdx.x / H_kv) * (TOK * U) + threadIdx.x / 64 * (32 / L) + threadIdx.x % 32 / L;
    const long long stride = which ? v_stride : k_stride;
    const uint16_t* from = (which ? V : K) + head * D + l * 16 + tok0 * stride;
    const int rest = (int)min(n_tokens - tok0, (long long)TOK * U);  // tokens of the block from this lane's first on
    const int32_t* slots = slot + tok0;
    int at[U];
    uint4 raw[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        at[u] = -1;
        raw[u][0] = raw[u][1] = make_uint4(0, 0, 0, 0);
        if (u * TOK < rest) {
            at[u] = slots[u * TOK];
            raw[u][0] = reinterpret_cast<const uint4*>(from)[0];
            raw[u][1] = reinterpret_cast<const uint4*>(from)[1];
        }
        from += TOK * stride;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t in[8] = {raw[u][0].x, raw[u][0].y, raw[u][0].z, raw[u][0].w, raw[u][1].x, raw[u][1].y, raw[u][1].z, raw[u][1].w};
        uint32_t w[2];
        const uint32_t pair = kv4_quantise<D>(in, which, l, w);
        if (at[u] < 0 || at[u] >= n_slots) continue;
        kv4_put<D>(pages + ((size_t)(at[u] / KV4_PAGE) * H_kv + head) * kv4_head_bytes(D), which, at[u] % KV4_PAGE, l, w, pair);
    }
}

template <int D, int U>
__global__ void __launch_bounds__(KS_THREADS) k_kv4_load(const uint8_t* pages, long long n_slots, int H_kv, uint16_t* K,
                                                         uint16_t* V, long long n_tokens, long long k_stride, long long v_stride,
                                                         const int32_t* slot) {
    dep_wait();
    dep_release();
    constexpr int L = D / 16, TOK = KS_THREADS / 2 / L;
    const int l = threadIdx.x % L, which = threadIdx.x / 32 & 1;    // a warp has rows of K or rows of V
    const int head = blockIdx.x % H_kv;
    const long long tok0 = (long long)(blockIdx.x / H_kv) * (TOK * U) + threadIdx.x / 64 * (32 / L) + threadIdx.x % 32 / L;
    const long long stride = which ? v_stride : k_stride;
    uint16_t* to = (which ? V : K) + head * D + l * 16 + tok0 * stride;
    const int rest = (int)min(n_tokens - tok0, (long long)TOK * U);
    const int32_t* slots = slot + tok0;
    int at[U];
    uint32_t w[U][2], pair[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        at[u] = u * TOK < rest ? slots[u * TOK] : -1;
        if (at[u] >= n_slots) at[u] = -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        w[u][0] = w[u][1] = pair[u] = 0;
        if (at[u] >= 0) {
            const uint8_t* block = pages + ((size_t)(at[u] / KV4_PAGE) * H_kv + head) * kv4_head_bytes(D);
            const int r = at[u] % KV4_PAGE;
            if (which == 0) {
                const uint8_t* from = block + kv4_k_word<D>(r, l >> 1, 2 * (l & 1));
                w[u][0] = *reinterpret_cast<const uint32_t*>(from);
                w[u][1] = *reinterpret_cast<const uint32_t*>(from + D / 8);
            } else if (D == 128) {
                const uint2 two = *reinterpret_cast<const uint2*>(block + kv4_v_word<D>(r, 0, l));
                w[u][0] = two.x;
                w[u][1] = two.y;
            } else {
                const uint32_t a = *reinterpret_cast<const uint32_t*>(block + kv4_v_word<D>(r, 0, l));
                const uint32_t b = *reinterpret_cast<const uint32_t*>(block + kv4_v_word<D>(r, 0, 4 + l));
                w[u][0] = __byte_perm(a, b, 0x5410);
                w[u][1] = __byte_perm(a, b, 0x7632);
            }
            pair[u] = *reinterpret_cast<const uint32_t*>(block + kv4_scale_word<D>(which, r, l >> 1));
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        uint32_t c[2] = {w[u][0], w[u][1]};
        if (which) {
            c[0] = kv4_transpose<D / 16, 1>(c[0], l);
            c[1] = kv4_transpose<D / 16, 1>(c[1], l);
        }
        uint16_t* row = to;
        to += TOK * stride;
        if (at[u] < 0) continue;
        // two elements at a time, i and i + 4: bf16 0x4300 | u is 128 + u; u and s u + b in bf16, the latter rounded once
        const uint32_t s2 = __byte_perm(pair[u], 0, 0x1010), b2 = __byte_perm(pair[u], 0, 0x3232);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint32_t v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t c128 = ((c[k] >> (4 * i)) & 0x000f000fu) | 0x43004300u;
                asm("{\n .reg .b32 t;\n add.rn.bf16x2 t, %1, %2;\n fma.rn.bf16x2 %0, t, %3, %4;\n}" : "=r"(v[i]) : "r"(c128), "r"(0xC300C300u), "r"(s2), "r"(b2));
            }
            reinterpret_cast<uint4*>(row)[k] = make_uint4(__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410), __byte_perm(v[0], v[1], 0x7632),
                                                          __byte_perm(v[2], v[3], 0x7632));
        }
    }
}

// ---- page tables ------------------------------------------------------------------------------------------------------
constexpr int KT_THREADS = 1024;
constexpr int KT_MAX = AG_KV4_MAX_ROWS;              // requests of one call: one thread each
constexpr int KT_SCAN = 8;                           // runs of 32 counts that a warp has in flight as it walks over the pages
constexpr int KT_SEGMENTS = 4096;                    // stretches of pages that compaction counts by: of 32 pages up to 131072 of them
// Up to so many slots are written by the allocating block itself, more by a second launch: 2048 slots take 10.2 to 11.1 us in all against 10.4 to
// 11.7, 4096 13.1 to 13.6 against 11.0 to 13.4 (8, 128 and 1024 rows; 65536 pages).
constexpr int KT_INLINE_TOKENS = 2048;

// exclusive sum over the block of one value per thread; *total = the sum
template <class T>
__device__ __forceinline__ T block_scan(T v, T* warp_sum, T* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    T inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T u = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += u;
    }
    __syncthreads();                                 // warp_sum may still be read from the scan before
    if (lane == 31) warp_sum[warp] = inc;
    __syncthreads();
    if (warp == 0) {
        T s = warp_sum[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const T u = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += u;
        }
        warp_sum[lane] = s;
    }
    __syncthreads();
    *total = warp_sum[31];
    return inc - v + (warp ? warp_sum[warp - 1] : 0);
}

struct TableArgs {
    int32_t *page_of, *len, *refs;
    int n_rows, max_pages, n_pages;
};

// Request i (thread i) wants need[i] pages; free pages are dealt in ascending order to the requests in order, request i getting the
// ranks before[i] .. before[i] + need[i] - 1.  A request is granted when all of them exist; one that needs none always is (a token in a page that the
// row owns does not wait for another row's page).  Ends with the pages entered in the
// tables (column first[i] on) and counted.  Returns whether this thread's request is granted.
// Every warp walks over its thirty-second of the pages, neighbouring lanes at neighbouring counts: 128 rows grow in 4.2 us among 2048 pages,
// 7.5 among 65536 (39 with neighbouring counts in one thread's hands).
struct GrantShared {
    long long warp_sum64[32];
    long long before[KT_MAX];                        // 64 bits: 1024 requests of up to 2^25 pages each
    int warp_sum[32];
    int need[KT_MAX], first[KT_MAX], row[KT_MAX];
};
__device__ inline bool grant_pages(const TableArgs& t, int n, int need, int first, int row, GrantShared* sh) {
    long long total_need;
    int total_free;
    const long long before = block_scan((long long)need, sh->warp_sum64, &total_need);
    sh->before[threadIdx.x] = before;
    sh->need[threadIdx.x] = need;
    sh->first[threadIdx.x] = first;
    sh->row[threadIdx.x] = row;
    const int lane = threadIdx.x & 31, seg = (t.n_pages + KT_THREADS - 1) / KT_THREADS * 32;
    const int p0 = (int)min((long long)(threadIdx.x >> 5) * seg, (long long)t.n_pages), p1 = min(p0 + seg, t.n_pages);
    int mine = 0;
    for (int p = p0 + lane; p < p1; p += 32 * KT_SCAN) {
        int refs[KT_SCAN];
#pragma unroll
        for (int u = 0; u < KT_SCAN; ++u) refs[u] = p + 32 * u < p1 ? t.refs[p + 32 * u] : 1;
#pragma unroll
        for (int u = 0; u < KT_SCAN; ++u) mine += refs[u] <= 0;
    }
    int rank = block_scan(mine, sh->warp_sum, &total_free);       // (its barriers also publish before, need, first, row)
    rank = __shfl_sync(0xffffffffu, rank, 0);                     // free pages in front of the warp's
    for (int p = p0; p < p1 && rank < total_need; p += 32 * KT_SCAN) {
        int refs[KT_SCAN];
#pragma unroll
        for (int u = 0; u < KT_SCAN; ++u) refs[u] = p + 32 * u + lane < p1 ? t.refs[p + 32 * u + lane] : 1;
#pragma unroll
        for (int u = 0; u < KT_SCAN; ++u) {
            const unsigned open = __ballot_sync(0xffffffffu, refs[u] <= 0);
            const int at = rank + __popc(open & ((1u << lane) - 1u));
            rank += __popc(open);
            if (refs[u] > 0 || at >= total_need) continue;
            int a = 0, b = n - 1;                                   // the last request with before <= at
            while (a < b) {
                const int m = (a + b + 1) >> 1;
                if (sh->before[m] <= at) a = m; else b = m - 1;
            }
            const int k = (int)(at - sh->before[a]);
            if (k < sh->need[a] && sh->before[a] + sh->need[a] <= total_free) {
                t.page_of[(size_t)sh->row[a] * t.max_pages + sh->first[a] + k] = p + 32 * u + lane;
                t.refs[p + 32 * u + lane] = 1;
            }
        }
    }
    return need == 0 || before + need <= total_free;
}

// Whether request i is the first of the call that names `key` (a row; -1: none).  Open addressing in shared memory, twice as many places as requests.
struct FirstShared {
    int key[2 * KT_MAX], first[2 * KT_MAX];
};
__device__ inline bool is_first(int key, FirstShared* sh) {
    for (int i = threadIdx.x; i < 2 * KT_MAX; i += KT_THREADS) {
        sh->key[i] = -1;
        sh->first[i] = KT_MAX;
    }
    __syncthreads();
    uint32_t at = 0;
    if (key >= 0) {
        at = (uint32_t)key * 2654435761u >> 21;                            // 11 bits
        static_assert(2 * KT_MAX == 1 << 11, "places of the table");
        for (int tries = 0; tries < 2 * KT_MAX; ++tries, at = (at + 1) & (2 * KT_MAX - 1)) {
            const int seen = atomicCAS(&sh->key[at], -1, key);
            if (seen == -1 || seen == key) break;
        }
        atomicMin(&sh->first[at], (int)threadIdx.x);
    }
    __syncthreads();
    return key >= 0 && sh->first[at] == (int)threadIdx.x;
}

// slot of token j: request i with new_off[i] <= j < new_off[i + 1], position len - new + j - new_off[i] (len: after the call)
__device__ __forceinline__ int slot_of(const TableArgs& t, const int32_t* row, const int32_t* new_off, const int32_t* ok, int n, int j) {
    if (j < new_off[0] || j >= new_off[n]) return -1;
    int a = 0, b = n - 1;
    while (a < b) {
        const int m = (a + b + 1) >> 1;
        if (new_off[m] <= j) a = m; else b = m - 1;
    }
    if (!ok[a] || j >= new_off[a + 1]) return -1;
    const int r = row[a];
    const int pos = t.len[r] - (new_off[a + 1] - j);
    if (pos < 0) return -1;
    const int page = t.page_of[(size_t)r * t.max_pages + pos / KV4_PAGE];
    return page >= 0 && page < t.n_pages ? page * KV4_PAGE + pos % KV4_PAGE : -1;
}

__global__ void __launch_bounds__(KT_THREADS) k_kv4_extend(const TableArgs t, const int32_t* row, const int32_t* new_off,
                                                           int n, int32_t* slot, int inline_tokens, int32_t* ok) {
    __shared__ union { GrantShared grant; FirstShared first; } sh;
    dep_wait();
    dep_release();
    const int i = threadIdx.x;
    int r = i < n ? row[i] : -1;
    const bool first_time = is_first(r, &sh.first);                        // a row named twice: only the first time counts
    int need = 0, first = 0;
    long long len0 = 0, fresh = 0;
    if (i < n) {
        fresh = (long long)new_off[i + 1] - new_off[i];
        bool fine = first_time && r < t.n_rows && fresh >= 0 && new_off[i] >= 0;
        if (fine) {
            len0 = t.len[r];
            fine = len0 >= 0 && len0 + fresh <= (long long)t.max_pages * KV4_PAGE;
        }
        if (fine) {
            first = (int)((len0 + KV4_PAGE - 1) / KV4_PAGE);
            need = (int)((len0 + fresh + KV4_PAGE - 1) / KV4_PAGE) - first;
        } else {
            r = -1;
        }
    }
    __syncthreads();
    const bool granted = grant_pages(t, n, need, first, r, &sh.grant) && r >= 0;
    if (granted) t.len[r] = (int)(len0 + fresh);
    if (i < n) ok[i] = granted ? 1 : 0;
    __syncthreads();                                                       // tables and ok are complete for this block
    for (int j = i; j < inline_tokens; j += KT_THREADS) slot[j] = slot_of(t, row, new_off, ok, n, j);
}

__global__ void __launch_bounds__(256) k_kv4_slots(const TableArgs t, const int32_t* row, const int32_t* new_off, int n,
                                                   int32_t* slot, int n_tokens, const int32_t* ok) {
    dep_wait();
    dep_release();
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j < n_tokens) slot[j] = slot_of(t, row, new_off, ok, n, j);
}

__global__ void __launch_bounds__(KT_THREADS) k_kv4_fork_plan(const TableArgs t, const int32_t* src, const int32_t* dst,
                                                              int n, int32_t* ok) {
    __shared__ union { GrantShared grant; FirstShared first; } sh;
    dep_wait();
    dep_release();
    const int i = threadIdx.x;
    int r = i < n ? dst[i] : -1;
    const bool first_time = is_first(r, &sh.first);
    int need = 0, first = 0, len = 0;
    if (i < n) {
        const int s = src[i];
        bool fine = first_time && r < t.n_rows && s >= 0 && s < t.n_rows && s != r;
        if (fine) {
            len = t.len[s];
            fine = t.len[r] == 0 && len >= 0 && (long long)len <= (long long)t.max_pages * KV4_PAGE;
        }
        if (fine) {
            first = len / KV4_PAGE;
            need = len % KV4_PAGE > 0;
        } else {
            r = -1;
        }
    }
    __syncthreads();
    const bool granted = grant_pages(t, n, need, first, r, &sh.grant) && r >= 0;
    if (granted) t.len[r] = len;                                           // every thread has read its lengths (barriers in grant_pages)
    if (i < n) ok[i] = granted ? 1 : 0;
}

// copies `units` pieces of 16 bytes, a block's threads side by side, four loads in flight a thread
__device__ __forceinline__ void copy16(uint4* to, const uint4* from, int units) {
    int i = threadIdx.x;
    const int step = blockDim.x;
    for (; i + 3 * step < units; i += 4 * step) {
        const uint4 a = from[i], b = from[i + step], c = from[i + 2 * step], d = from[i + 3 * step];
        to[i] = a;
        to[i + step] = b;
        to[i + 2 * step] = c;
        to[i + 3 * step] = d;
    }
    for (; i < units; i += step) to[i] = from[i];
}

// block (request, part): part 0 also shares the full pages; every part copies its share of the open page
__global__ void __launch_bounds__(256) k_kv4_fork_copy(const TableArgs t, const int32_t* src, const int32_t* dst,
                                                       const int32_t* ok, uint8_t* pages, size_t page_bytes, int parts) {
    dep_wait();
    dep_release();
    const int i = blockIdx.x / parts, part = blockIdx.x - i * parts;
    if (!ok[i]) return;
    const int r = dst[i], len = t.len[r];
    const int32_t* from = t.page_of + (size_t)src[i] * t.max_pages;
    int32_t* to = t.page_of + (size_t)r * t.max_pages;
    const int full = len / KV4_PAGE;
    if (part == 0) {
        for (int c = threadIdx.x; c < full; c += blockDim.x) {
            const int p = from[c];
            to[c] = p;
            if (p >= 0 && p < t.n_pages) atomicAdd(&t.refs[p], 1);
        }
    }
    if (len % KV4_PAGE) {
        const int a = from[full], b = to[full];
        if (a < 0 || a >= t.n_pages || b < 0 || b >= t.n_pages) return;
        const int units = (int)(page_bytes / 16), u0 = (int)((long long)units * part / parts), u1 = (int)((long long)units * (part + 1) / parts);
        copy16(reinterpret_cast<uint4*>(pages + (size_t)b * page_bytes) + u0, reinterpret_cast<const uint4*>(pages + (size_t)a * page_bytes) + u0, u1 - u0);
    }
}

// a page is given back by whoever takes it out of the table, so that a row named twice gives it back once
__global__ void __launch_bounds__(256) k_kv4_free(const TableArgs t, const int32_t* row) {
    dep_wait();
    dep_release();
    const int r = row[blockIdx.x];
    if (r < 0 || r >= t.n_rows) return;
    int32_t* entry = t.page_of + (size_t)r * t.max_pages;
    for (int c = threadIdx.x; c < t.max_pages; c += blockDim.x) {
        if (entry[c] < 0) continue;
        const int p = atomicExch(&entry[c], -1);
        if (p >= 0 && p < t.n_pages) atomicSub(&t.refs[p], 1);
    }
    if (threadIdx.x == 0) t.len[r] = 0;
}

// Where every page goes: with n_used pages in use, the k-th used page from n_used on takes the k-th free page below.  What is counted is the
// used pages in front of a segment of 32 pages (a multiple in large pools): a free page's number among the holes is the free pages in front of it, a
// mover's number is the used pages in front of it less those below n_used.  The holes are listed first, then every mover reads its own.
// Plan and move of 65536 pages that are in place already: 28 us (238 with neighbouring counts in one thread's hands); of a million pages of 5 KB, half of
// them in use at random: 1270 us, 760 of them copies; of four million: 5.0 ms (each mover walking through a segment for its hole: 7.7 and 88 ms).
__global__ void __launch_bounds__(KT_THREADS) k_kv4_compact_plan(const TableArgs t, int32_t* moved) {
    __shared__ int warp_sum[32];
    __shared__ int used_before[KT_SEGMENTS];
    __shared__ uint32_t used_mask[KT_SEGMENTS];                            // with segments of 32 pages
    dep_wait();
    dep_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int words = (t.n_pages + 31) / 32;
    const bool small = words <= KT_SEGMENTS;
    const int seg_words = small ? 1 : ((words + KT_SEGMENTS - 1) / KT_SEGMENTS + KT_SCAN - 1) / KT_SCAN * KT_SCAN;
    const int seg = 32 * seg_words, n_seg = (words + seg_words - 1) / seg_words;
    const int per_warp = small ? KT_SCAN : 1;                              // segments that a warp takes at a time
    for (int a = threadIdx.x; a < KT_SEGMENTS; a += KT_THREADS) used_before[a] = 0;
    __syncthreads();
    for (int a0 = warp * per_warp; a0 < n_seg; a0 += 32 * per_warp)
        for (int i = 0; i < seg_words; i += KT_SCAN) {
            const int p = a0 * seg + 32 * i + lane;
            int refs[KT_SCAN];
#pragma unroll
            for (int u = 0; u < KT_SCAN; ++u) refs[u] = p + 32 * u < t.n_pages ? t.refs[p + 32 * u] : 0;
#pragma unroll
            for (int u = 0; u < KT_SCAN; ++u) {
                const uint32_t mask = __ballot_sync(0xffffffffu, refs[u] > 0);
                const int a = small ? a0 + u : a0;
                if (lane == 0 && a < n_seg) {
                    used_before[a] += __popc(mask);
                    used_mask[a] = mask;
                }
            }
        }
    __syncthreads();
    constexpr int PER = KT_SEGMENTS / KT_THREADS;
    int c[PER], sum = 0, n_used;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        c[i] = used_before[threadIdx.x * PER + i];
        sum += c[i];
    }
    sum = block_scan(sum, warp_sum, &n_used);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        used_before[threadIdx.x * PER + i] = sum;
        sum += c[i];
    }
    __syncthreads();
    int used_below = 0;                                                    // used pages below n_used, which stay
    for (int p = n_used / seg * seg + lane; p < n_used; p += 32) used_below += t.refs[p] > 0;
    used_below = __reduce_add_sync(0xffffffffu, used_below) + (n_used < t.n_pages ? used_before[n_used / seg] : n_used);
    // pages lo .. hi - 1 (and others of their segments): f(page, in use?, used pages in front of it)
    auto walk = [&](int lo, int hi, auto&& f) {
        for (int a = lo / seg + warp; a < n_seg && a * seg < hi; a += 32) {
            int before = used_before[a];
            for (int i = 0; i < seg_words; i += KT_SCAN) {
                const int p = a * seg + 32 * i + lane;
                int refs[KT_SCAN];
                if (!small)
#pragma unroll
                    for (int u = 0; u < KT_SCAN; ++u) refs[u] = p + 32 * u < t.n_pages ? t.refs[p + 32 * u] : 0;
#pragma unroll
                for (int u = 0; u < KT_SCAN; ++u) {
                    if (small && u > 0) break;
                    const uint32_t mask = small ? used_mask[a] : __ballot_sync(0xffffffffu, refs[u] > 0);
                    f(p + 32 * u, mask >> lane & 1u, before + __popc(mask & ((1u << lane) - 1u)));
                    before += __popc(mask);
                }
            }
        }
    };
    // the list of holes takes the front of `moved` for a while: there are no more of them than pages below n_used
    if (used_below < n_used)
        walk(0, n_used, [&](int p, bool used, int in_front) {
            if (!used && p < n_used) moved[p - in_front] = p;
        });
    __syncthreads();
    walk(n_used, t.n_pages, [&](int p, bool used, int in_front) {
        if (p >= n_used && p < t.n_pages) moved[p] = used ? moved[in_front - used_below] : -1;
    });
    __syncthreads();
    walk(0, n_used, [&](int p, bool used, int) {
        if (p < n_used) moved[p] = used ? p : -1;
    });
}

// Copies page from[i] (from = NULL: i) to page to[i], in parts; pairs with a page outside the pool, or of a page with itself, are passed over.  A
// block's threads look for work side by side, as most pages of a large pool stay where they are.  With `refs` the pages' counts move too.
__device__ __forceinline__ void copy_pages(const int32_t* from, const int32_t* to, long long n, long long n_pages,
                                           uint8_t* pages, size_t page_bytes, int parts, int32_t* refs) {
    __shared__ int work_from[256], work_to[256], work_part[256], n_found;
    const int units = (int)(page_bytes / 16);
    const long long n_work = n * parts;
    for (long long w0 = blockIdx.x; w0 < n_work; w0 += (long long)gridDim.x * 256) {
        if (threadIdx.x == 0) n_found = 0;
        __syncthreads();
        const long long w = w0 + (long long)threadIdx.x * gridDim.x;
        if (w < n_work) {
            const long long i = w / parts, a = from ? from[i] : i, b = to[i];
            if (a >= 0 && a < n_pages && b >= 0 && b < n_pages && a != b) {
                const int k = atomicAdd(&n_found, 1);                      // (in any order: the copies are independent)
                work_from[k] = (int)a;
                work_to[k] = (int)b;
                work_part[k] = (int)(w - i * parts);
            }
        }
        __syncthreads();
        for (int k = 0; k < n_found; ++k) {
            const int a = work_from[k], b = work_to[k], part = work_part[k];
            const int u0 = (int)((long long)units * part / parts), u1 = (int)((long long)units * (part + 1) / parts);
            copy16(reinterpret_cast<uint4*>(pages + (size_t)b * page_bytes) + u0, reinterpret_cast<const uint4*>(pages + (size_t)a * page_bytes) + u0, u1 - u0);
            if (refs && part == 0 && threadIdx.x == 0) {
                refs[b] = refs[a];
                refs[a] = 0;
            }
        }
        __syncthreads();                                                   // the list has been read
    }
}

// page (and its count) by page, and the tables, entry by entry
__global__ void __launch_bounds__(256) k_kv4_compact_move(const TableArgs t, const int32_t* moved, uint8_t* pages,
                                                          size_t page_bytes, int parts) {
    dep_wait();
    dep_release();
    const long long n_entries = (long long)t.n_rows * t.max_pages, step = (long long)gridDim.x * blockDim.x;
    for (long long e = (long long)blockIdx.x * blockDim.x + threadIdx.x; e < n_entries; e += step) {
        const int p = t.page_of[e];
        if (p >= 0) t.page_of[e] = p < t.n_pages ? moved[p] : -1;
    }
    copy_pages(nullptr, moved, t.n_pages, t.n_pages, pages, page_bytes, parts, t.refs);
}

__global__ void __launch_bounds__(256) k_kv4_copy(const int32_t* from, const int32_t* to, long long n, long long n_pages,
                                                  uint8_t* pages, size_t page_bytes, int parts) {
    dep_wait();
    dep_release();
    copy_pages(from, to, n, n_pages, pages, page_bytes, parts, nullptr);
}

static bool misaligned(const int32_t* a, const int32_t* b = nullptr, const int32_t* c = nullptr) {
    return ((uintptr_t)a | (uintptr_t)b | (uintptr_t)c) & 3u;
}

static TableArgs table_args(const ag_kv4_pool* pool, const ag_kv4_table* t) {
    return TableArgs{t->page_of, t->len, t->refs, t->n_rows, t->max_pages, (int)pool->n_pages};
}

}  // namespace ag

using namespace ag;

extern "C" size_t ag_kv4_page_bytes(int H_kv, int D) {
    if (H_kv < 1 || H_kv > 1024 || (D != 64 && D != 128)) return 0;
    return (size_t)H_kv * kv4_head_bytes(D);
}

static ag_status kv4_rows(bool store, const ag_kv4_pool* pool, const void* K, const void* V, int64_t n_tokens, int64_t k_stride, int64_t v_stride,
                          const int32_t* slot, void* cuda_stream) {
    if (!kv4_pool_ok(pool) || n_tokens < 0 || n_tokens > (1ll << 31) - 1) return AG_ERR_ARG;
    if (n_tokens == 0) return AG_OK;
    const int64_t width = (int64_t)pool->H_kv * pool->D;
    if (!K || !V || !slot || (((uintptr_t)K | (uintptr_t)V) & 15u) || ((uintptr_t)slot & 3u) || k_stride < width || v_stride < width || (k_stride % 8) || (v_stride % 8))
        return AG_ERR_ARG;
    // several rows a lane once that leaves two rounds of blocks for 148 SMs
    const int one = KS_THREADS / 2 / (pool->D / 16);
    const bool many = n_tokens * pool->H_kv >= 2ll * 148 * 8 * KS_ROWS * one;
    const int block_tokens = one * (many ? KS_ROWS : 1);
    const long long blocks = (n_tokens + block_tokens - 1) / block_tokens * pool->H_kv;
    if (blocks > 0x7fffffffll) return AG_ERR_ARG;
    ag_status st = check_arch();
    if (st != AG_OK) return st;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    const long long n_slots = (long long)pool->n_pages * KV4_PAGE;
    uint8_t* pages = (uint8_t*)pool->pages;
    if (store) {
        auto kernel = pool->D == 128 ? (many ? k_kv4_store<128, KS_ROWS> : k_kv4_store<128, 1>) : (many ? k_kv4_store<64, KS_ROWS> : k_kv4_store<64, 1>);
        AG_CUDA(launch_dependent(kernel, (unsigned)blocks, KS_THREADS, stream, pages, n_slots, pool->H_kv, (const uint16_t*)K, (const uint16_t*)V, n_tokens, k_stride, v_stride, slot));
    } else {
        auto kernel = pool->D == 128 ? (many ? k_kv4_load<128, KS_ROWS> : k_kv4_load<128, 1>) : (many ? k_kv4_load<64, KS_ROWS> : k_kv4_load<64, 1>);
        AG_CUDA(launch_dependent(kernel, (unsigned)blocks, KS_THREADS, stream, pages, n_slots, pool->H_kv, (uint16_t*)const_cast<void*>(K),
                                 (uint16_t*)const_cast<void*>(V), n_tokens, k_stride, v_stride, slot));
    }
    count_launch();
    return AG_OK;
}

extern "C" ag_status ag_kv4_store(const ag_kv4_pool* pool, const void* K, const void* V, int64_t n_tokens, int64_t k_stride, int64_t v_stride,
                                  const int32_t* slot, void* cuda_stream) {
    return kv4_rows(true, pool, K, V, n_tokens, k_stride, v_stride, slot, cuda_stream);
}

extern "C" ag_status ag_kv4_load(const ag_kv4_pool* pool, const int32_t* slot, int64_t n_tokens, void* K, void* V, int64_t k_stride, int64_t v_stride,
                                 void* cuda_stream) {
    return kv4_rows(false, pool, K, V, n_tokens, k_stride, v_stride, slot, cuda_stream);
}

extern "C" ag_status ag_kv4_extend(const ag_kv4_pool* pool, const ag_kv4_table* table, const int32_t* row, const int32_t* new_off, int n, int32_t* slot,
                                   int64_t n_tokens, int32_t* ok, void* cuda_stream) {
    if (!kv4_pool_ok(pool) || !kv4_table_ok(table) || n < 0 || n > KT_MAX || n_tokens < 0 || n_tokens > (1ll << 31) - 1) return AG_ERR_ARG;
    if (n == 0 && n_tokens == 0) return AG_OK;
    if (!row || !new_off || !ok || (n_tokens > 0 && !slot) || n == 0 || misaligned(row, new_off, ok) || misaligned(slot)) return AG_ERR_ARG;
    ag_status st = check_arch();
    if (st != AG_OK) return st;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    const TableArgs t = table_args(pool, table);
    const bool one = n_tokens <= KT_INLINE_TOKENS;
    AG_CUDA(launch_dependent(k_kv4_extend, 1, KT_THREADS, stream, t, row, new_off, n, slot, one ? (int)n_tokens : 0, ok));
    count_launch();
    if (!one) {
        AG_CUDA(launch_dependent(k_kv4_slots, (unsigned)((n_tokens + 255) / 256), 256, stream, t, row, new_off, n, slot, (int)n_tokens, ok));
        count_launch();
    }
    return AG_OK;
}

extern "C" ag_status ag_kv4_fork(const ag_kv4_pool* pool, const ag_kv4_table* table, const int32_t* src, const int32_t* dst, int n, int32_t* ok,
                                 void* cuda_stream) {
    if (!kv4_pool_ok(pool) || !kv4_table_ok(table) || n < 0 || n > KT_MAX) return AG_ERR_ARG;
    if (n == 0) return AG_OK;
    if (!src || !dst || !ok || misaligned(src, dst, ok)) return AG_ERR_ARG;
    ag_status st = check_arch();
    if (st != AG_OK) return st;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    const TableArgs t = table_args(pool, table);
    const size_t page_bytes = ag_kv4_page_bytes(pool->H_kv, pool->D);
    AG_CUDA(launch_dependent(k_kv4_fork_plan, 1, KT_THREADS, stream, t, src, dst, n, ok));
    count_launch();
    const int parts = (int)std::max<size_t>(1, page_bytes / 16384);       // a block copies 16 to 32 KB
    AG_CUDA(launch_dependent(k_kv4_fork_copy, (unsigned)(n * parts), 256, stream, t, src, dst, (const int32_t*)ok, (uint8_t*)pool->pages, page_bytes, parts));
    count_launch();
    return AG_OK;
}

extern "C" ag_status ag_kv4_free(const ag_kv4_pool* pool, const ag_kv4_table* table, const int32_t* row, int n, void* cuda_stream) {
    if (!kv4_pool_ok(pool) || !kv4_table_ok(table) || n < 0 || n > KT_MAX) return AG_ERR_ARG;
    if (n == 0) return AG_OK;
    if (!row || misaligned(row)) return AG_ERR_ARG;
    ag_status st = check_arch();
    if (st != AG_OK) return st;
    AG_CUDA(launch_dependent(k_kv4_free, (unsigned)n, 256, reinterpret_cast<cudaStream_t>(cuda_stream), table_args(pool, table), row));
    count_launch();
    return AG_OK;
}

extern "C" ag_status ag_kv4_compact(const ag_kv4_pool* pool, const ag_kv4_table* table, int32_t* moved, void* cuda_stream) {
    if (!kv4_pool_ok(pool) || !kv4_table_ok(table) || !moved || ((uintptr_t)moved & 3u)) return AG_ERR_ARG;
    ag_status st = check_arch();
    if (st != AG_OK) return st;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    const TableArgs t = table_args(pool, table);
    const size_t page_bytes = ag_kv4_page_bytes(pool->H_kv, pool->D);
    AG_CUDA(launch_dependent(k_kv4_compact_plan, 1, KT_THREADS, stream, t, moved));
    count_launch();
    const int parts = (int)std::max<size_t>(1, page_bytes / 16384);
    const long long work = std::max((long long)t.n_pages * parts, ((long long)t.n_rows * t.max_pages + 255) / 256);
    AG_CUDA(launch_dependent(k_kv4_compact_move, (unsigned)std::min<long long>(work, 148 * 8), 256, stream, t, (const int32_t*)moved, (uint8_t*)pool->pages,
                             page_bytes, parts));
    count_launch();
    return AG_OK;
}

extern "C" ag_status ag_kv4_copy(const ag_kv4_pool* pool, const int32_t* from, const int32_t* to, int64_t n, void* cuda_stream) {
    if (!kv4_pool_ok(pool) || n < 0 || n > pool->n_pages) return AG_ERR_ARG;
    if (n == 0) return AG_OK;
    if (!to || (((uintptr_t)to | (uintptr_t)from) & 3u)) return AG_ERR_ARG;
    ag_status st = check_arch();
    if (st != AG_OK) return st;
    const size_t page_bytes = ag_kv4_page_bytes(pool->H_kv, pool->D);
    const int parts = (int)std::max<size_t>(1, page_bytes / 16384);
    AG_CUDA(launch_dependent(k_kv4_copy, (unsigned)std::min<long long>(n * parts, 148 * 8), 256, reinterpret_cast<cudaStream_t>(cuda_stream), from, to, (long long)n,
                             (long long)pool->n_pages, (uint8_t*)pool->pages, page_bytes, parts));
    count_launch();
    return AG_OK;
}
