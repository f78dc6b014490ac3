// Attention of drafted tokens over the 4-bit cache and over one another (a tree): see include/asymgemm.h, "drafted tokens".
//
// Work unit = (request, KV head, up to 256 rows), a row being a (token, head of the group) pair: all rows of a unit share every key.  A unit's keys are tiles of 128:
// tile 0 the drafted tokens themselves (64 at most), tile t two pages of the cache.  With 128 rows and 128 keys a tile is
//     S = Q K^T              tcgen05.mma, 128 x 128 x D, fp16 operands, scores in tensor memory
//     P = 2^(S - m)          one thread a row; P as fp16 back into tensor memory, over the scores
//     O += P V               tcgen05.mma with the A operand in tensor memory
// Two tiles are in flight, w = 0, 1, each with scores, statistics and outputs of its own:
//     more than 128 rows     w = half of the rows, both see every key tile: keys and values are decoded once for 256 rows
//     up to 128 rows         w = parity of the key tile
//     up to 64 (32) rows     besides, the 128 lanes hold the rows twice (four times), each copy has one half (quarter) of the tile's keys and zeros as the other
//                            probabilities: the MMAs cost the same, the exponentials a half (a quarter)
// and the statistics and outputs of all copies are put together at the end of the unit.
//
// Codes become fp16 operands in shared memory: a nibble in the lowest (or next) four bits of a half is the subnormal u 2^-24 (u 2^-20), and one multiply-add
// with s 2^24 (s 2^20) and the base gives s u + b, rounded once.  For that a tile's values are taken at a power of two that puts the largest below 2^-5: K's for every
// tile on its own (scores are multiplied back with the row's factor), V's for the run of a unit (outputs move when it grows).  Inside a chunk of eight operand elements
// the order is that of the nibbles, (0, 4), (1, 5), (2, 6), (3, 7); Q is laid out the same, and V's columns are put back when the outputs are written.
//
// All tiles of all units stand in one line that is cut into equal runs, one per block: uneven lengths, one long request or many short ones are the same case.  Units that
// two or more blocks share leave parts (normalised outputs, maximum, sum) in the workspace, which a second launch puts together.
//
// 640 threads: warps 0-7 softmax and epilogue (two groups of four), 8 MMA, 9 units and copies of keys, 10 exponents, 11 copies of values, 12-19 decoding, half of them of keys, half of values.
//
// Bound: a tile takes some 6360 warp instructions (decoding 2000, softmax 2500, the rest the roles' bookkeeping) on five warps a scheduler, 2500 cycles (2230 with D = 64); its MMAs take 1300, its
// exponentials 1024, its bytes 500.  4 requests x 32 tokens x 32 heads over 131072 keys: 319 us at 1.965 GHz (840 TFLOP/s), 370 when it is repeated for seconds (the chip is at its 1000 W
// then and runs at 1.68 GHz).  Code that runs once a unit costs the fetching of its instructions, six cycles each, so it is loops wherever it can be: with the unit's end written out
// (88 KB of code in all; 86 now, 9 of them for drafts out of the ordinary, which few calls fetch) 64 requests over 200 to 4000 keys took 123 us, now 87 to 88.
// Other splits, measured: 16 softmax warps, two threads a row (4 requests as above 372 us against 341 of that time); tiles handed on in halves of 64 keys (418 against 405: QK^T with 64
// columns takes an MMA as long as with 128); more operand stages where they fit, D = 64 (no difference).
#include <math.h>
#include <string.h>

#include <algorithm>

#include "kv4.cuh"

namespace ag {

constexpr int TA_TILE = 128;
// stages: operands; raw codes of K and of V, each with one copying warp and one group of decoders (in a ring that both share, one copying warp could come round twice before the other's
// stage had been read); raw (scale, base) pairs
constexpr int TA_OPS = 3, TA_KCODES = 3, TA_VCODES = 2, TA_CODES = TA_KCODES + TA_VCODES, TA_SCALES = 4;
constexpr int TA_INFO = 8, TA_UNITS = 4;
constexpr int TA_SOFT = 8, TA_DECODERS = 8;                // warps
constexpr int TA_THREADS = 640;
constexpr int TA_READERS = TA_SOFT + TA_DECODERS + 3;      // warps that read a unit: and MMA, exponents, values' copies
constexpr int TA_REGS_SOFT = 112, TA_REGS_OTHER = 80;      // 256 x 112 + 384 x 80 <= 640 x 96
constexpr int TA_BLOCKS = 148;
// Places of the line that a unit takes beside its tiles, for Q, drafts and its end: measured, five to six tiles' time (64 requests over 200 to 4000 keys 86.7 us, with 4 of them 90.1, with 2
// 96.6), and even, since tiles of more than 128 rows take two places (16 trees of 40 to 64 tokens 83.0 us, with 5 95.6).  None where every tile can have a block of its own, since
// then the longest run counts, not the sum (with it, a short request's tiles would be handled one after the other by a few blocks).
constexpr int TA_UNIT = 6;
// The reference m of a row moves when its maximum is more than 2^11.5 times as large, and P is taken times 2^4: at most 2^15.5, and 2^-25 is lost of it, 2^-29 of the largest.  m is a whole number
// (2^m at most the maximum when it moves), so that what there is by then (sums, outputs, the tile's probabilities so far) is multiplied by a power of two and loses no more than that.  (With 2^5 and 2^10 2^-35 was lost, but one tile in
// three had a row to move, whose outputs are multiplied and written back while everybody waits: 4 trees over 131072 tokens 371 us instead of 325.)
constexpr uint32_t TA_WAIT = 1;                            // turns of the clock (2.2 to 4.4 s) that a role waits for a barrier: a wait lasts some tiles, microseconds
constexpr float TA_LAZY = 11.5f, TA_SHIFT = 4.f;

struct TreeArgs {
    const uint16_t *Q, *K, *V;
    uint16_t* O;
    const uint8_t* pages;
    long long q_stride, k_stride, v_stride, o_stride;
    const int32_t *row, *off, *parent, *page_of, *len;
    int H_q, H_kv, G, n_seq, n_rows, max_pages, n_pages, n_tokens, max_tokens, most_len, part_rows;
    uint32_t by_g;                         // 2^32 / G, rounded up (G > 1)
    float scale_log2e;
    int32_t* status;
    struct TreeCross* cross;               // [blocks]: the unit that begins in block i and goes on beyond it
    float2* stats;                         // [2 blocks][part_rows]
    float* part;                           // [2 blocks][part_rows][D]
};
struct TreeCross {
    long long begin, quota;                // place of the unit's first tile in the line; tiles of a run
    int weight, tiles, token0, row0, rows, head, unit_places, pad;
};

struct TreeUnit {
    int token0, n;                         // the request's first drafted token, their number
    int row0, rows;                        // of the request's rows
    int len, table_row, head;
    int tile0, tile1, tiles;               // this block's tiles, the unit's
    int two, copies, buf;                  // rows in both halves; log2 of the copies of the rows; buffer of Q (two: both)
    int slot;                              // part slot, -1: the whole unit is here
    int stop, pad;
};
constexpr int TA_ODD = 1, TA_WIDE = 2;     // a drafted value is not in the products; drafts are so unequal that large ones are taken on their own
struct alignas(16) TreeInfo {
    int ek, ev, v0, v1, odd;               // exponents of K and V; keys that count in the tile's halves; of drafts: TA_ODD, TA_WIDE
};

struct TreeCtl {
    uint64_t q_full[2], q_empty[2], op_full[TA_OPS], op_empty[TA_OPS], codes_full[TA_CODES], codes_empty[TA_CODES];
    uint64_t scales_full[TA_SCALES], scales_ready[TA_SCALES], scales_empty[TA_SCALES];
    uint64_t s_full[2], p_full[2], pv_done[2], unit_full[TA_UNITS], unit_empty[TA_UNITS], together, drain;
    unsigned long long sees[2][AG_TREE_MAX];
    float row_scale[2][TA_TILE];
    float2 stats[2 * TA_TILE], sums[2 * TA_TILE];          // of a lane's row: its own part's (maximum, sum); all parts'
    uint32_t draft_top[TA_UNITS][AG_TREE_MAX];             // WIDE: largest finite element of a large drafted key, as bf16; 0: the key has the tile's exponent
    unsigned long long big[TA_UNITS];                      // WIDE: drafted tokens whose values stay out of the products
    TreeUnit unit[TA_UNITS];
    TreeInfo info[TA_INFO];
    int valid[TA_INFO][2];
    long long warp_sum[TA_THREADS / 32][2];
    long long total, start_before;
    uint32_t tmem_base;
    int abort_flag, start_seq, odd, ev[TA_SOFT];
};

template <int D>
struct TCfg {
    static constexpr int op_bytes = TA_TILE * D * 2;       // a tile of operands, and of Q
    static constexpr int code_bytes = 2 * 32 * D;          // K's or V's codes of two pages
    static constexpr int scale_bytes = 2 * 16 * D;         // K's and V's pairs of two pages
    static constexpr int smem_bytes = (2 + TA_OPS) * op_bytes + TA_CODES * code_bytes + TA_SCALES * scale_bytes + (int)((sizeof(TreeCtl) + 127) / 128 * 128) + 1024;
};
static_assert(TCfg<128>::smem_bytes <= 227 * 1024, "does not fit");
constexpr int TA_MIN_SMEM = 120 * 1024;                    // one block an SM: it takes all of the tensor memory

__device__ __forceinline__ float pow2i(int k) { return __uint_as_float((uint32_t)(127 + k) << 23); }     // -126 .. 127
// v 2^k for any k of -250 .. 250
__device__ __forceinline__ float times_pow2(float v, int k) { return v * pow2i(k >> 1) * pow2i(k - (k >> 1)); }

// Eight codes of a word times scales plus bases, as four pairs (0, 4), (1, 5), (2, 6), (3, 7): a (scales 2^24 and 2^20, bases) for the first two, b for the others.
struct Scale2 {
    uint32_t s24, s20, base;
};
__device__ __forceinline__ uint4 decode_word(uint32_t w, const Scale2& a, const Scale2& b) {
    const uint32_t v = w >> 8;
    return make_uint4(fma_f16x2(w & 0x000f000fu, a.s24, a.base), fma_f16x2(w & 0x00f000f0u, a.s20, a.base), fma_f16x2(v & 0x000f000fu, b.s24, b.base),
                      fma_f16x2(v & 0x00f000f0u, b.s20, b.base));
}
// k24 = 2^(24 - exponent): scales and bases of two groups side by side
__device__ __forceinline__ Scale2 scale_pair(uint32_t lo, uint32_t hi, float k24) {
    const float k20 = k24 * 0.0625f, k0 = k20 * 0x1p-20f;
    const float s0 = bf16_lo(lo), s1 = bf16_lo(hi);
    return Scale2{pack_f16(s0 * k24, s1 * k24), pack_f16(s0 * k20, s1 * k20), pack_f16(bf16_hi(lo) * k0, bf16_hi(hi) * k0)};
}

// exponent under which a drafted key is taken: a large one's own, or the tile's
__device__ __forceinline__ int key_exponent(uint32_t top, int ek) { return top ? min((int)(top >> 7) - 127 + 6, 133) : ek; }
// what a row sees of a drafted value that is not in the products: with the probability p of a token whose value is large, 0 otherwise
__device__ __forceinline__ float left_out(float p, float v) { return fabsf(v) < INFINITY ? (p == 0.f ? 0.f : p * v) : v; }

// A request: its drafted tokens, cached tokens and places in the line.
struct TreeSeq {
    int first, n, rows, len, table_row, tiles, weight;     // weight: of all units of a head, a unit of more than 128 rows counting twice
    __device__ __forceinline__ int units() const { return (rows + 255) / 256; }
    __device__ __forceinline__ int per_head(int unit_places) const { return weight * tiles + units() * unit_places; }     // (below 2^30)
};
__device__ __forceinline__ TreeSeq tree_seq(const TreeArgs& x, int s) {
    TreeSeq r;
    const int first = min(max(x.off[s], 0), x.n_tokens), stop = min(max(x.off[s + 1], first), x.n_tokens);
    r.first = first;
    r.n = min(stop - first, x.max_tokens);
    r.rows = r.n * x.G;
    r.table_row = x.row ? x.row[s] : s;
    r.len = r.table_row >= 0 && r.table_row < x.n_rows ? min(max(x.len[r.table_row], 0), x.most_len) : 0;
    r.tiles = (int)((r.len + (TA_TILE - 1u)) / TA_TILE) + 1;
    const int rest = r.rows % 256;
    r.weight = r.rows / 256 * 2 + (rest > 128 ? 2 : rest > 0 ? 1 : 0);
    return r;
}
// a / b, without the division of 64 bits where the numbers are small (some 600 cycles, and most of a small call's first 3 us are like these)
__device__ __forceinline__ long long quotient(long long a, long long b) { return (a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b); }
// token of a request's row (below 4096; G at most 64)
__device__ __forceinline__ int token_of(const TreeArgs& x, int row) { return x.G == 1 ? row : (int)__umulhi((uint32_t)row, x.by_g); }
// tiles of the unit at place `begin` of the line that lie in front of `place`
__device__ __forceinline__ int tiles_before(long long place, long long begin, int unit_places, int weight, int tiles) {
    const int d = (int)min(max(place - begin, 0ll), 1ll << 30);
    return min(max((d - unit_places + weight - 1) >> (weight - 1), 0), tiles);      // (weight: 1 or 2)
}

template <int D>
__global__ void __launch_bounds__(TA_THREADS, 1) k_attn_tree_kv4(const TreeArgs x) {
    using C = TCfg<D>;
    constexpr int NG = D / 32;
    extern __shared__ uint8_t tree_smem[];
    uint8_t* smem = tree_smem + ((1024 - (smem_u32(tree_smem) & 1023)) & 1023);
    uint8_t* q_smem = smem;
    uint8_t* op_smem = q_smem + 2 * C::op_bytes;
    uint8_t* code_smem = op_smem + TA_OPS * C::op_bytes;
    uint8_t* scale_smem = code_smem + TA_CODES * C::code_bytes;
    TreeCtl* ctl = reinterpret_cast<TreeCtl*>(scale_smem + TA_SCALES * C::scale_bytes);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;      // (from one lane: known to be the same for the warp)

    if (tid == 0) {
        ctl->abort_flag = 0;
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&ctl->q_full[i]), TA_DECODERS);
            mbar_init(smem_u32(&ctl->q_empty[i]), TA_SOFT);
            mbar_init(smem_u32(&ctl->s_full[i]), 2);
            mbar_init(smem_u32(&ctl->p_full[i]), 4);
            mbar_init(smem_u32(&ctl->pv_done[i]), 1);
        }
        for (int i = 0; i < TA_OPS; ++i) {
            mbar_init(smem_u32(&ctl->op_full[i]), TA_DECODERS / 2);
            mbar_init(smem_u32(&ctl->op_empty[i]), 1);
        }
        for (int i = 0; i < TA_CODES; ++i) {
            mbar_init(smem_u32(&ctl->codes_full[i]), 1);
            mbar_init(smem_u32(&ctl->codes_empty[i]), TA_DECODERS / 2);
        }
        for (int i = 0; i < TA_SCALES; ++i) {
            mbar_init(smem_u32(&ctl->scales_full[i]), 1);
            mbar_init(smem_u32(&ctl->scales_ready[i]), 1);
            mbar_init(smem_u32(&ctl->scales_empty[i]), TA_DECODERS);
        }
        for (int i = 0; i < TA_UNITS; ++i) {
            mbar_init(smem_u32(&ctl->unit_full[i]), 1);
            mbar_init(smem_u32(&ctl->unit_empty[i]), TA_READERS);
        }
        mbar_init(smem_u32(&ctl->together), TA_SOFT);
        mbar_init(smem_u32(&ctl->drain), 1);
        mbar_fence_init();
    }
    if (warp == 8) {
        tmem_alloc(smem_u32(&ctl->tmem_base), 512);
        tmem_relinquish();
    }
    dep_wait();
    dep_release();

    // ---- the block's run of the line
    const int per = (x.n_seq + TA_THREADS - 1) / TA_THREADS, s0 = min(tid * per, x.n_seq), s1 = min(s0 + per, x.n_seq);
    long long mine = 0, mine_units = 0;            // places of tiles, units
#pragma unroll 1
    for (int s = s0; s < s1; ++s) {
        const TreeSeq q = tree_seq(x, s);
        mine += (long long)q.per_head(0) * x.H_kv;
        mine_units += (long long)q.units() * x.H_kv;
    }
    long long inc = mine, inc_units = mine_units;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long up = __shfl_up_sync(0xffffffffu, inc, o), up_units = __shfl_up_sync(0xffffffffu, inc_units, o);
        if (lane >= o) {
            inc += up;
            inc_units += up_units;
        }
    }
    if (lane == 31) {
        ctl->warp_sum[warp][0] = inc;
        ctl->warp_sum[warp][1] = inc_units;
    }
    __syncthreads();
    long long before = inc - mine, total = 0, before_units = inc_units - mine_units, total_units = 0;
#pragma unroll 1
    for (int w = 0; w < (min(x.n_seq, TA_THREADS) + 31) / 32; ++w) {           // (the other warps have no request)
        const long long a = ctl->warp_sum[w][0], b = ctl->warp_sum[w][1];
        if (w < warp) {
            before += a;
            before_units += b;
        }
        total += a;
        total_units += b;
    }
    const int unit_places = total <= (long long)gridDim.x ? 0 : TA_UNIT;
    total += total_units * unit_places;
    before += before_units * unit_places;
    mine += mine_units * unit_places;
    const long long quota = max(quotient(total + gridDim.x - 1, gridDim.x), 1ll);
    const long long p0 = min(quota * blockIdx.x, total), p1 = min(p0 + quota, total);
    if (p0 < p1 && before <= p0 && p0 < before + mine) {
        long long at = before;
        int s = s0;
#pragma unroll 1
        for (; s < s1; ++s) {
            const long long l = (long long)tree_seq(x, s).per_head(unit_places) * x.H_kv;
            if (p0 < at + l) break;
            at += l;
        }
        ctl->start_seq = s;
        ctl->start_before = at;
    }
    if (tid == 0) {
        if (blockIdx.x == 0) *x.status = AG_OK;
        x.cross[blockIdx.x].rows = 0;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctl->tmem_base;
    bool ok = true;
    // Every wait is bounded, in time; who has given up waits no more.  (Few instructions: there are some thirty of them, and twenty warps in eight roles share the instruction caches.)
    auto wait = [&](uint64_t* b, uint32_t parity) -> bool {
        ok = __all_sync(0xffffffffu, mbar_wait_clock(smem_u32(b), parity, TA_WAIT));
        return ok;
    };
    // unit u, which stays where it is until every reader has left it
    auto next_unit = [&](uint32_t u) -> bool { return wait(&ctl->unit_full[u % TA_UNITS], (u / TA_UNITS) & 1) && !ctl->unit[u % TA_UNITS].stop; };
    auto leave_unit = [&](uint32_t u) {
        __syncwarp();
        if (elect_one()) mbar_arrive(smem_u32(&ctl->unit_empty[u % TA_UNITS]));
    };

    if (warp >= TA_SOFT) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(TA_REGS_OTHER));
    uint32_t n_tile = 0, n_code = 0;               // tiles, and tiles with codes, before the unit in hand
    // the stage of the c-th tile of codes, of K (which = 0) or V, and its turn's parity
    auto code_stage_of = [&](int which, uint32_t c, uint32_t& parity) -> uint32_t {
        const uint32_t turn = which ? c / TA_VCODES : c / TA_KCODES;
        parity = turn & 1;
        return which ? TA_KCODES + c - turn * TA_VCODES : c - turn * TA_KCODES;
    };
    // copies of a unit's pages: warp 9 K's codes and all pairs (which = 0), warp 11 V's codes (1)
    auto copies = [&](int which, const TreeUnit& un) {
        const int nt = un.tile1 - un.tile0, drafts = un.tile0 == 0, len = un.len;
        const uint8_t* heads = x.pages + (size_t)un.head * kv4_head_bytes(D);
        const int32_t* pages = x.page_of + (size_t)max(un.table_row, 0) * x.max_pages;
        int window = -1, page = -1;                // pages of 16 tiles in the lanes: lane l has page 32 window + l of the row
#pragma unroll 1
        for (int j = 0; j < nt; ++j) {
            const uint32_t n = n_tile + j;
            const int t = un.tile0 + j, c = 2 * (t - 1);
            if (which == 0 && !wait(&ctl->scales_empty[n % TA_SCALES], ((n / TA_SCALES) & 1) ^ 1)) return;
            if (t == 0) {                          // the drafted tokens: nothing to copy
                if (which == 0 && elect_one()) {
                    ctl->valid[n % TA_INFO][0] = min(un.n, 64);
                    ctl->valid[n % TA_INFO][1] = 0;
                    mbar_arrive(smem_u32(&ctl->scales_full[n % TA_SCALES]));
                }
                __syncwarp();
                continue;
            }
            if (c >> 5 != window) {
                window = c >> 5;
                page = window * 32 + lane < (len + 63) / 64 ? pages[window * 32 + lane] : -1;
            }
            uint32_t turn;
            const uint32_t stage = code_stage_of(which, n_code + j - drafts, turn);
            if (!wait(&ctl->codes_empty[stage], turn ^ 1)) return;
            const int id0 = __shfl_sync(0xffffffffu, page, c & 31), id1 = __shfl_sync(0xffffffffu, page, (c + 1) & 31);
            const int v0 = id0 >= 0 && id0 < x.n_pages ? min(max(len - 64 * c, 0), 64) : 0, v1 = id1 >= 0 && id1 < x.n_pages ? min(max(len - 64 * c - 64, 0), 64) : 0;
            if (elect_one()) {
                const uint32_t bar = smem_u32(&ctl->codes_full[stage]), sbar = smem_u32(&ctl->scales_full[n % TA_SCALES]);
                const uint32_t to = smem_u32(code_smem + stage * C::code_bytes), sto = smem_u32(scale_smem + (n % TA_SCALES) * C::scale_bytes);
                const int there = (v0 > 0) + (v1 > 0);
                const uint8_t *p0 = heads + (size_t)max(id0, 0) * x.H_kv * kv4_head_bytes(D), *p1 = heads + (size_t)max(id1, 0) * x.H_kv * kv4_head_bytes(D);
                if (which == 0) {
                    ctl->valid[n % TA_INFO][0] = v0;
                    ctl->valid[n % TA_INFO][1] = v1;
                    mbar_expect_tx(sbar, there * 16 * D);
                    if (v0 > 0) bulk_load(sto, p0 + 64 * D, 16 * D, sbar);
                    if (v1 > 0) bulk_load(sto + 16 * D, p1 + 64 * D, 16 * D, sbar);
                }
                mbar_expect_tx(bar, there * 32 * D);
                if (v0 > 0) bulk_load(to, p0 + which * 32 * D, 32 * D, bar);
                if (v1 > 0) bulk_load(to + 32 * D, p1 + which * 32 * D, 32 * D, bar);
            }
            __syncwarp();
        }
        n_tile += nt;
        n_code += nt - drafts;
    };
    if (warp == 9) {
        // ------------------------------------------------ units; copies of keys
        uint32_t u = 0, toggle = 0;
        long long at = ctl->start_before;
        int s = p0 < p1 ? ctl->start_seq : x.n_seq;
#pragma unroll 1
        while (ok && s < x.n_seq && at < p1) {
            const TreeSeq q = tree_seq(x, s);
            const long long line = (long long)q.per_head(unit_places) * x.H_kv;
            const int per_head = q.per_head(unit_places);
            const int units = q.units();
#pragma unroll 1
            for (int h = at < p0 && line > 0 ? (int)quotient(p0 - at, per_head) : 0; ok && h < x.H_kv && line > 0; ++h) {
                if (at + (long long)h * per_head >= p1) break;
#pragma unroll 1
                for (int i = 0; ok && i < units; ++i) {
                    const long long begin = at + (long long)h * per_head + i * (2 * q.tiles + unit_places);
                    const int rows = min(q.rows - i * 256, 256), weight = rows > 128 ? 2 : 1;
                    const int t0 = tiles_before(p0, begin, unit_places, weight, q.tiles), t1 = tiles_before(p1, begin, unit_places, weight, q.tiles);
                    if (t0 >= t1) continue;
                    if (!wait(&ctl->unit_empty[u % TA_UNITS], ((u / TA_UNITS) & 1) ^ 1)) break;
                    const int two = rows > 128, buf = two ? 0 : (int)(toggle & 1);
                    toggle += two ? 0 : 1;
                    if (lane == 0) {
                        TreeUnit r;
                        r.token0 = q.first; r.n = q.n; r.row0 = i * 256; r.rows = rows; r.len = q.len; r.table_row = q.table_row; r.head = h;
                        r.tile0 = t0; r.tile1 = t1; r.tiles = q.tiles; r.two = two; r.copies = rows <= 32 ? 2 : rows <= 64 ? 1 : 0; r.buf = buf;
                        r.slot = t0 == 0 && t1 == q.tiles ? -1 : 2 * (int)blockIdx.x + (t1 < q.tiles ? 1 : 0);
                        r.stop = 0; r.pad = 0;
                        ctl->unit[u % TA_UNITS] = r;
                        mbar_arrive(smem_u32(&ctl->unit_full[u % TA_UNITS]));
                        if (t0 == 0 && t1 < q.tiles) {
                            TreeCross c;
                            c.begin = begin; c.quota = quota; c.weight = weight; c.tiles = q.tiles; c.token0 = q.first; c.row0 = i * 256; c.rows = rows; c.head = h;
                            c.unit_places = unit_places; c.pad = 0;
                            x.cross[blockIdx.x] = c;
                        }
                    }
                    __syncwarp();
                    ++u;
                    copies(0, ctl->unit[(u - 1) % TA_UNITS]);
                    if (!ok) break;
                }
            }
            at += line;
            ++s;
        }
        if (ok && wait(&ctl->unit_empty[u % TA_UNITS], ((u / TA_UNITS) & 1) ^ 1) && lane == 0) {
            ctl->unit[u % TA_UNITS].stop = 1;
            mbar_arrive(smem_u32(&ctl->unit_full[u % TA_UNITS]));
        }
        __syncwarp();
    } else if (warp == 10) {
        // ------------------------------------------------ exponents of the tiles
        // the largest |base| + 15 s of this lane's tokens among those of a tile that count, of K and of V
        auto coded_tops = [&](uint32_t n, int v0, int v1, float (&top)[2]) {
#pragma unroll 1
            for (int k = 0; k < 4; ++k) {
                const int tok = (k & 1) * 32 + lane;
                if (tok >= (k >> 1 ? v1 : v0)) continue;
                const uint8_t* at = scale_smem + (n % TA_SCALES) * C::scale_bytes + (k >> 1) * 16 * D + tok * 4 * NG;
#pragma unroll
                for (int which = 0; which < 2; ++which)
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        const uint32_t pair = reinterpret_cast<const uint32_t*>(at + which * 8 * D)[g];
                        top[which] = fmaxf(top[which], fmaf(15.f, fabsf(bf16_lo(pair)), fabsf(bf16_hi(pair))));
                    }
            }
        };
#pragma unroll 1
        for (uint32_t u = 0; next_unit(u); ++u) {
            const TreeUnit& un = ctl->unit[u % TA_UNITS];
            int ev = 1000;                                         // none yet
#pragma unroll 1
            for (int j = 0; j < un.tile1 - un.tile0; ++j) {
                const uint32_t n = n_tile + j;
                if (!wait(&ctl->scales_full[n % TA_SCALES], (n / TA_SCALES) & 1)) break;
                const int v0 = ctl->valid[n % TA_INFO][0], v1 = ctl->valid[n % TA_INFO][1];
                float top[2] = {0.f, 0.f};
                int odd = 0;
                if (un.tile0 + j == 0) {
                    // the largest magnitudes by their bits, two elements of a word side by side; four pieces of 16 bytes of K and of V in flight
                    uint32_t most[2] = {0, 0}, first = 0;                       // (first: of this lane's piece of the first token, K's high, V's low)
                    const int pieces = un.n * (D / 8);
                    int up[2];                                                  // parents (on their way meanwhile)
#pragma unroll
                    for (int k = 0; k < 2; ++k) up[k] = lane + 32 * k < un.n && x.parent ? x.parent[un.token0 + lane + 32 * k] : lane + 32 * k - 1;
#pragma unroll 1
                    for (int i0 = lane; i0 < pieces; i0 += 128) {
                        uint4 raw[8];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int i = i0 + 32 * q < pieces ? i0 + 32 * q : i0, d = un.head * D + i % (D / 8) * 8;
                            raw[q] = *reinterpret_cast<const uint4*>(x.K + (un.token0 + (long long)(i / (D / 8))) * x.k_stride + d);
                            raw[4 + q] = *reinterpret_cast<const uint4*>(x.V + (un.token0 + (long long)(i / (D / 8))) * x.v_stride + d);
                        }
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            const uint32_t m = __vmaxu2(__vmaxu2(raw[q].x & 0x7fff7fffu, raw[q].y & 0x7fff7fffu), __vmaxu2(raw[q].z & 0x7fff7fffu, raw[q].w & 0x7fff7fffu));
                            most[q >> 2] = __vmaxu2(most[q >> 2], m);
                            if ((q & 3) == 0 && i0 < D / 8) first |= max(m & 0xffffu, m >> 16) << (q ? 0 : 16);
                        }
                    }
                    uint32_t all[2], of_first[2];
#pragma unroll
                    for (int which = 0; which < 2; ++which) {
                        all[which] = __reduce_max_sync(0xffffffffu, max(most[which] & 0xffffu, most[which] >> 16));
                        of_first[which] = __reduce_max_sync(0xffffffffu, which ? first & 0xffffu : first >> 16);
                        top[which] = __uint_as_float(all[which] << 16);
                    }
                    // A draft may be far larger than what the rows that do not see it see (a branch gone astray, padding, another tree), or not finite.  Such a key is taken under a power of two of its
                    // own, such a value stays out of the products: rows that see it get it at the end of the unit.  Every row sees a token without a parent, and one such token alone, finite, not 0,
                    // and no draft above 2^6 times as large: nothing to do.
                    constexpr uint32_t room = 6 << 7;                              // 2^6 in the bits of a bf16
                    unsigned long long roots = 0;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int i = lane + 32 * k;
                        roots |= (unsigned long long)__ballot_sync(0xffffffffu, i < un.n && !(up[k] >= 0 && up[k] < i)) << (32 * k);
                    }
                    if (roots != 1 || max(all[0], all[1]) >= 0x7f80u || !of_first[0] || !of_first[1] || all[0] > of_first[0] + room || all[1] > of_first[1] + room) {
                        uint32_t* tops = ctl->draft_top[u % TA_UNITS];
                        // the largest finite magnitudes of every token, K's in the high half, V's in the low
                        bool not_finite = false;
#pragma unroll 1
                        for (int i0 = 0; i0 < pieces; i0 += 32) {
                            const int i = i0 + lane, t = i / (D / 8), d = un.head * D + i % (D / 8) * 8;
                            uint32_t m = 0;
#pragma unroll
                            for (int which = 0; which < 2; ++which) {
                                uint4 raw = make_uint4(0, 0, 0, 0);
                                if (i < pieces) raw = *reinterpret_cast<const uint4*>(which ? x.V + (un.token0 + (long long)t) * x.v_stride + d : x.K + (un.token0 + (long long)t) * x.k_stride + d);
                                const uint32_t w[4] = {raw.x & 0x7fff7fffu, raw.y & 0x7fff7fffu, raw.z & 0x7fff7fffu, raw.w & 0x7fff7fffu};
                                uint32_t top2 = 0;
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    const uint32_t not_here = __vcmpgtu2(w[k], 0x7f7f7f7fu);
                                    not_finite |= which && not_here;
                                    top2 = __vmaxu2(top2, w[k] & ~not_here);
                                }
                                m |= max(top2 & 0xffffu, top2 >> 16) << (which ? 0 : 16);
                            }
#pragma unroll
                            for (int o = 1; o < D / 8; o <<= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
                            if (i < pieces && lane % (D / 8) == 0) tops[t] = m;
                        }
                        __syncwarp();
                        const uint32_t t0 = lane < un.n ? tops[lane] : 0, t1 = lane + 32 < un.n ? tops[lane + 32] : 0;
                        const uint32_t k0 = t0 >> 16, k1 = t1 >> 16, w0 = t0 & 0xffffu, w1 = t1 & 0xffffu;
                        auto least = [&](uint32_t a, uint32_t b, bool zeros) { return __reduce_min_sync(0xffffffffu, min(a || zeros ? a : 0xffffu, b || zeros ? b : 0xffffu)); };
                        // What all rows see at least.  Keys: the smallest that is not 0 (a row of scores 0 has no use for an exponent).  Values: the smallest without a parent, or what the cached
                        // tile behind this one holds, if there is one; where neither has anything, the smallest that is not 0, or, if cached ones may follow, nothing.
                        const uint32_t least_key = least(k0, k1, false);
                        const bool r0 = roots >> lane & 1, r1 = roots >> (lane + 32) & 1;
                        uint32_t least_value = least(r0 ? w0 : 0xffffu, r1 ? w1 : 0xffffu, true);
                        if (un.tile1 > 1) {
                            if (!wait(&ctl->scales_full[(n + 1) % TA_SCALES], ((n + 1) / TA_SCALES) & 1)) break;
                            float cached[2] = {0.f, 0.f};
                            coded_tops(n + 1, ctl->valid[(n + 1) % TA_INFO][0], ctl->valid[(n + 1) % TA_INFO][1], cached);
                            least_value = max(least_value, __reduce_max_sync(0xffffffffu, __float_as_uint(cached[1])) >> 16);
                        } else if (least_value == 0) {
                            least_value = least(w0, w1, false);
                        }
                        const uint32_t key_limit = least_key + room, limit = least_value ? least_value + room : 0;
                        const unsigned long long big = __ballot_sync(0xffffffffu, w0 > limit) | (unsigned long long)__ballot_sync(0xffffffffu, w1 > limit) << 32;
                        if (lane == 0) ctl->big[u % TA_UNITS] = big;
                        __syncwarp();
                        tops[lane] = k0 > key_limit ? k0 : 0;
                        tops[lane + 32] = k1 > key_limit ? k1 : 0;
                        top[0] = __uint_as_float(max(k0 > key_limit ? 0u : k0, k1 > key_limit ? 0u : k1) << 16);
                        top[1] = __uint_as_float(max(w0 > limit ? 0u : w0, w1 > limit ? 0u : w1) << 16);
                        if (not_finite || big) odd = TA_WIDE | TA_ODD;
                        else if (k0 > key_limit || k1 > key_limit || all[0] >= 0x7f80u) odd = TA_WIDE;
                    }
                } else {
                    coded_tops(n, v0, v1, top);
                }
                int e[2];
#pragma unroll
                for (int which = 0; which < 2; ++which) {
                    const uint32_t bits = __reduce_max_sync(0xffffffffu, __float_as_uint(top[which]));
                    e[which] = bits == 0 ? -1000 : min(max((int)(bits >> 23) - 127 + 6, -100), 133);
                }
                odd = (int)__reduce_or_sync(0xffffffffu, (unsigned)odd);
                __syncwarp();
                if (e[1] > -1000 && (ev == 1000 || e[1] > ev)) ev = min(e[1] + 2, 133);     // (two binades of room, so that it seldom grows)
                if (lane == 0) {
                    TreeInfo& f = ctl->info[n % TA_INFO];
                    f.ek = e[0] == -1000 ? 0 : e[0];
                    f.ev = ev == 1000 ? 0 : ev;
                    f.v0 = v0; f.v1 = v1; f.odd = odd;
                    mbar_arrive(smem_u32(&ctl->scales_ready[n % TA_SCALES]));
                }
                __syncwarp();
            }
            n_tile += un.tile1 - un.tile0;
            if (!ok) break;
            leave_unit(u);
        }
    } else if (warp == 11) {
        // ------------------------------------------------ copies of values; before them, tokens beyond the most that a request may have
#pragma unroll 1
        for (int s = blockIdx.x; s < x.n_seq; s += gridDim.x) {
            const int first = min(max(x.off[s], 0), x.n_tokens), stop = min(max(x.off[s + 1], first), x.n_tokens);
#pragma unroll 1
            for (int t = first + x.max_tokens; t < stop; ++t)
#pragma unroll 1
                for (int d = lane * 8; d < x.H_q * D; d += 256) *reinterpret_cast<uint4*>(x.O + (long long)t * x.o_stride + d) = make_uint4(0, 0, 0, 0);
        }
#pragma unroll 1
        for (uint32_t u = 0; next_unit(u); ++u) {
            copies(1, ctl->unit[u % TA_UNITS]);
            if (!ok) break;
            leave_unit(u);
        }
    } else if (warp == 8) {
        // ------------------------------------------------ MMA issuer (the warp runs converged, one elected lane issues)
        const uint32_t idesc_s = make_idesc_f16(TA_TILE, TA_TILE, 0, 0), idesc_o = make_idesc_f16(TA_TILE, D, 0, 1);
        const uint64_t dk_t = make_smem_desc(0, 16, 1024, 2);                  // Q, K: K-major, 128-byte swizzle
        const uint64_t dv_t = make_smem_desc(0, TA_TILE * 128, 1024, 2);       // V: N-major, 64-column blocks 16 KB apart
        const uint32_t q_base = smem_u32(q_smem), op_base = smem_u32(op_smem);
        uint32_t n_op = 0, q_parity = 0, p_parity = 0;      // parities: a bit for each barrier
        auto commit = [&](uint64_t* b) {
            if (elect_one()) tc_commit(smem_u32(b));
            __syncwarp();
        };
#pragma unroll 1
        for (uint32_t u = 0; next_unit(u); ++u) {
            const TreeUnit& un = ctl->unit[u % TA_UNITS];
            const int nt = __shfl_sync(0xffffffffu, un.tile1 - un.tile0, 0), two = __shfl_sync(0xffffffffu, un.two, 0), buf = __shfl_sync(0xffffffffu, un.buf, 0), lead = two ? 1 : 2;
#pragma unroll 1
            for (int b = 0; b < 2; ++b)
                if (two || buf == b) {
                    if (!wait(&ctl->q_full[b], q_parity >> b & 1)) break;
                    q_parity ^= 1u << b;
                }
            // step j: the products of V_j, the scores of K_{j + lead}, for one tile of rows or for both in turn; operands come in this order
#pragma unroll 1
            for (int j = -lead; j < nt && ok; ++j) {
                const bool pv = j >= 0, qk = j + lead < nt;
                const uint32_t nv = n_op, nk = n_op + (pv ? 1 : 0);
                n_op = nk + (qk ? 1 : 0);
                if (pv && !wait(&ctl->op_full[nv % TA_OPS], (nv / TA_OPS) & 1)) break;
                const int w0 = two ? 0 : j & 1, w1 = two ? 1 : j & 1;
#pragma unroll 1
                for (int w = w0; w <= w1; ++w) {
                    if (pv) {
                        if (!wait(&ctl->p_full[w], p_parity >> w & 1)) break;
                        p_parity ^= 1u << w;
                        tc_fence_after();
                        const uint64_t dv = dv_t | (uint64_t)__shfl_sync(0xffffffffu, (op_base + nv % TA_OPS * C::op_bytes) >> 4, 0);
                        const uint32_t first = j < lead ? 0u : 1u, d = tmem + 256 + w * D, p = tmem + w * TA_TILE;
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < TA_TILE / 16; ++k)                     // P of keys 64 h .. 64 h + 63 lies at columns 64 h .. 64 h + 31
                                tc_mma_f16_ts(d, p + (k >> 2) * 64 + (k & 3) * 8, dv + k * (2048 >> 4), idesc_o, k == 0 ? first : 1u);
                            tc_commit(smem_u32(&ctl->pv_done[w]));
                        }
                        __syncwarp();
                    }
                    if (qk) {
                        if (w == w0 && !wait(&ctl->op_full[nk % TA_OPS], (nk / TA_OPS) & 1)) break;
                        tc_fence_after();
                        const uint64_t dq = dk_t | (uint64_t)__shfl_sync(0xffffffffu, (q_base + (two ? w : buf) * C::op_bytes) >> 4, 0);
                        const uint64_t dk = dk_t | (uint64_t)__shfl_sync(0xffffffffu, (op_base + nk % TA_OPS * C::op_bytes) >> 4, 0);
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < D / 16; ++k)
                                tc_mma_f16(tmem + w * TA_TILE, dq + (k >> 2) * (TA_TILE * 128 >> 4) + (k & 3) * 2, dk + (k >> 2) * (TA_TILE * 128 >> 4) + (k & 3) * 2, idesc_s,
                                           k ? 1u : 0u);
                            tc_commit(smem_u32(&ctl->s_full[w]));
                            mbar_arrive(smem_u32(&ctl->s_full[w]));    // (with what this warp has seen: the tile's exponents, the rows' factors)
                        }
                        __syncwarp();
                    }
                }
                if (!ok) break;
                if (pv) commit(&ctl->op_empty[nv % TA_OPS]);
                if (qk) commit(&ctl->op_empty[nk % TA_OPS]);
            }
            if (!ok) break;
            leave_unit(u);
        }
        __syncwarp();
    } else {
        // ------------------------------------------------ decoders: Q, the drafted tokens and the cache's codes as operands
        // Whose operands a warp makes, K's or V's: those of one kind stand on the same schedulers, which then fetch the code of that kind only (64 requests 90.1 us at the time; with one of each on
        // every scheduler 91.8, the long cases alike)
        const int dwarp = warp - 12, which = dwarp >> 1 & 1;
        const int token = ((dwarp >> 2) * 2 + (dwarp & 1)) * 32 + lane, page = token >> 6, tk = token & 63, sw = token & 7;
        // Where the thread's codes are read and its operands written: K's run t (chunks t, 4 + t ..), V's words of elements 16 i' + 8 j' + h (chunks 2 h and 2 h + 1, or h), each with
        // t or h turned by the token so that neighbouring lanes meet no bank twice.  Operand row: chunk c at (c / 8) 16 KB + 128 row + 16 ((c ^ row) mod 8).
        const int turn = which == 0 ? (tk >> (D == 128 ? 1 : 2)) & 3 : D == 128 ? (tk >> 3) & 1 : (tk >> 3) & 3;
        const int src = page * 32 * D + (which == 0 ? tk * (D / 2) + turn * (D / 8) : (tk >> 3) * 4 * D + ((tk >> 1) & 3) * (D / 8) + (tk & 1) * (D / 16) + turn * (D / 2));
        const int dst = token * 128 + (((which && D == 128 ? 2 * turn : turn) ^ sw) & 7) * 16;
        uint32_t n_op = 0, q_parity = 0;
        auto arrive = [&](uint64_t* b) {
            __syncwarp();
            if (elect_one()) mbar_arrive(smem_u32(b));
        };
#pragma unroll 1
        for (uint32_t u = 0; next_unit(u); ++u) {
            const TreeUnit& un = ctl->unit[u % TA_UNITS];
            const int nt = un.tile1 - un.tile0, lead = un.two ? 1 : 2;
            // ---- Q: rows times a power of two that puts their largest element at 2^7
#pragma unroll 1
            for (int b = 0; b < 2; ++b) {
                if (!un.two && un.buf != b) continue;
                if (!wait(&ctl->q_empty[b], (q_parity >> b & 1) ^ 1)) break;
                q_parity ^= 1u << b;
                if (dwarp == TA_DECODERS - 1) {
                    // who sees whom among the drafted tokens: paths to the root by doubling, two tokens a lane
                    unsigned long long anc[2];
                    int jump[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int i = lane + 32 * k;
                        const int p = i < un.n ? x.parent ? x.parent[un.token0 + i] : i - 1 : -1;
                        jump[k] = p >= 0 && p < i ? p : -1;
                        anc[k] = 1ull << i;
                    }
#pragma unroll 1
                    while (__any_sync(0xffffffffu, jump[0] >= 0 || jump[1] >= 0)) {    // (a parent is in front of its child: six times at most)
                        unsigned long long more[2];
                        int far[2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const int j = max(jump[k], 0) & 31;
                            const unsigned long long a0 = __shfl_sync(0xffffffffu, anc[0], j), a1 = __shfl_sync(0xffffffffu, anc[1], j);
                            const int f0 = __shfl_sync(0xffffffffu, jump[0], j), f1 = __shfl_sync(0xffffffffu, jump[1], j);
                            more[k] = jump[k] < 0 ? 0 : jump[k] < 32 ? a0 : a1;
                            far[k] = jump[k] < 0 ? -1 : jump[k] < 32 ? f0 : f1;
                        }
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            anc[k] |= more[k];
                            jump[k] = far[k];
                        }
                    }
                    ctl->sees[b][lane] = anc[0];
                    ctl->sees[b][lane + 32] = anc[1];
                }
                constexpr int L = D / 8, R = 32 / L;               // lanes of a row, rows of a warp
                const int unit_row0 = un.two ? b * TA_TILE : 0, rows = min(un.rows - unit_row0, TA_TILE), distinct = TA_TILE >> un.copies;
                const int c = lane % L;
#pragma unroll 1
                for (int r0 = dwarp * R * 2; r0 < distinct; r0 += TA_DECODERS * R * 2) {
                    uint4 raw[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int r = r0 + k * R + lane / L, at = un.row0 + unit_row0 + r;
                        raw[k] = make_uint4(0, 0, 0, 0);
                        if (r < rows) raw[k] = *reinterpret_cast<const uint4*>(x.Q + (long long)(un.token0 + token_of(x, at)) * x.q_stride + (un.head * x.G + at - token_of(x, at) * x.G) * D + c * 8);
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int r = r0 + k * R + lane / L;
                        const uint32_t w[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
                        // the row's largest magnitude by its bits, two elements of a word side by side
                        uint32_t most = __vmaxu2(__vmaxu2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), __vmaxu2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
                        most = max(most & 0xffffu, most >> 16);
#pragma unroll
                        for (int o = 1; o < L; o <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
                        float top = __uint_as_float(most << 16);
                        if (__any_sync(0xffffffffu, most >= 0x7f80u)) {            // some are not finite: the largest of the others
                            top = 0.f;
#pragma unroll 1
                            for (int i = 0; i < 8; ++i) {
                                const uint32_t word = i < 4 ? i < 2 ? w[0] : w[1] : i < 6 ? w[2] : w[3];
                                const float v = fabsf(i & 1 ? bf16_hi(word) : bf16_lo(word));
                                if (v < INFINITY) top = fmaxf(top, v);
                            }
#pragma unroll 1
                            for (int o = 1; o < L; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                        }
                        float v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = i & 1 ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]);
                        const int shift = top == 0.f ? 0 : min(7 - ((int)(__float_as_uint(top) >> 23) - 127), 120);
                        const float f = pow2i(shift);
                        const uint4 out = make_uint4(pack_f16(v[0] * f, v[4] * f), pack_f16(v[1] * f, v[5] * f), pack_f16(v[2] * f, v[6] * f), pack_f16(v[3] * f, v[7] * f));
                        if (r < distinct) {
#pragma unroll 1
                            for (int to = r; to < TA_TILE; to += distinct)
                                *reinterpret_cast<uint4*>(q_smem + b * C::op_bytes + (c >> 3) * (TA_TILE * 128) + to * 128 + (((c ^ to) & 7) << 4)) = out;
                            if (c == 0) ctl->row_scale[b][r] = x.scale_log2e * pow2i(-shift);
                        }
                    }
                }
                fence_proxy_async_smem();
                arrive(&ctl->q_full[b]);
            }
            if (!ok) break;
            // ---- operands: four warps make K's, four V's; thread = token of the tile
            const int ahead = min(lead, nt), drafts = un.tile0 == 0;
            // the place among the unit's operands, which are made and used in the order K_0 .. K_{ahead - 1}, V_0 K_ahead V_1 K_{ahead + 1} .., the remaining V
            int place = which ? ahead : 0;
#pragma unroll 1
            for (int j = 0; j < nt; ++j) {
                const uint32_t n = n_tile + j;
                // the operand's stage, and the place of its codes
                if (j > 0) place += which ? (j <= nt - ahead ? 2 : 1) : (j < ahead ? 1 : 2);
                const uint32_t op = n_op + place, stage = op % TA_OPS, op_parity = (op / TA_OPS & 1) ^ 1;
                uint32_t code_parity;
                const uint32_t code_stage = code_stage_of(which, n_code + j - drafts, code_parity);
                if (!wait(&ctl->scales_ready[n % TA_SCALES], (n / TA_SCALES) & 1)) break;
                const TreeInfo& f = ctl->info[n % TA_INFO];
                const int e = which ? f.ev : f.ek;
                uint8_t* to = op_smem + stage * C::op_bytes;
                const bool coded = j > 0 || !drafts;
                if (coded) {
                    uint32_t pair[NG];
                    const uint8_t* sc = scale_smem + (n % TA_SCALES) * C::scale_bytes + page * 16 * D + which * 8 * D + tk * 4 * NG;
                    if (D == 128) *reinterpret_cast<uint4*>(pair) = *reinterpret_cast<const uint4*>(sc);
                    else *reinterpret_cast<uint2*>(pair) = *reinterpret_cast<const uint2*>(sc);
                    if (tk >= (page ? f.v1 : f.v0)) {
#pragma unroll
                        for (int g = 0; g < NG; ++g) pair[g] = 0;
                    }
                    const float k24 = pow2i(24 - e);
                    const uint8_t* codes = code_smem + code_stage * C::code_bytes;
                    if (which == 0) {
                        Scale2 g[NG];
#pragma unroll
                        for (int k = 0; k < NG; ++k) g[k] = scale_pair(pair[k], pair[k], k24);
                        if (!wait(&ctl->codes_full[code_stage], code_parity) || !wait(&ctl->op_empty[stage], op_parity)) break;
#pragma unroll 1
                        for (int t = 0; t < 4; ++t) {                                  // (t ^ turn: exclusive ors of the addresses' bits)
                            uint8_t *p = to + (dst ^ t * 16), *q = to + (dst ^ t * 16 ^ 64);
                            if (D == 128) {
                                const uint4 w = *reinterpret_cast<const uint4*>(codes + (src ^ t * 16));
                                *reinterpret_cast<uint4*>(p) = decode_word(w.x, g[0], g[0]);
                                *reinterpret_cast<uint4*>(q) = decode_word(w.y, g[1], g[1]);
                                *reinterpret_cast<uint4*>(p + TA_TILE * 128) = decode_word(w.z, g[NG - 2], g[NG - 2]);
                                *reinterpret_cast<uint4*>(q + TA_TILE * 128) = decode_word(w.w, g[NG - 1], g[NG - 1]);
                            } else {
                                const uint2 w = *reinterpret_cast<const uint2*>(codes + (src ^ t * 8));
                                *reinterpret_cast<uint4*>(p) = decode_word(w.x, g[0], g[0]);
                                *reinterpret_cast<uint4*>(q) = decode_word(w.y, g[1], g[1]);
                            }
                        }
                    } else {
                        const Scale2 a = D == 128 ? scale_pair(pair[0], pair[NG / 2], k24) : scale_pair(pair[0], pair[0], k24);
                        const Scale2 b = D == 128 ? scale_pair(pair[1], pair[NG - 1], k24) : scale_pair(pair[1], pair[1], k24);
                        if (!wait(&ctl->codes_full[code_stage], code_parity) || !wait(&ctl->op_empty[stage], op_parity)) break;
#pragma unroll 1
                        for (int h = 0; h < 4; ++h) {
                            uint8_t *p = to + (dst ^ h * (D == 128 ? 32 : 16)), *q = to + (dst ^ (D == 128 ? h * 32 ^ 16 : h * 16 ^ 64));
                            const uint8_t* from = codes + (src ^ h * (D / 2));
                            if (D == 128) {
                                const uint2 w = *reinterpret_cast<const uint2*>(from), y = *reinterpret_cast<const uint2*>(from + 2 * D);
                                *reinterpret_cast<uint4*>(p) = decode_word(w.x, a, b);
                                *reinterpret_cast<uint4*>(q) = decode_word(w.y, a, b);
                                *reinterpret_cast<uint4*>(p + TA_TILE * 128) = decode_word(y.x, a, b);
                                *reinterpret_cast<uint4*>(q + TA_TILE * 128) = decode_word(y.y, a, b);
                            } else {
                                *reinterpret_cast<uint4*>(p) = decode_word(*reinterpret_cast<const uint32_t*>(from), a, b);
                                *reinterpret_cast<uint4*>(q) = decode_word(*reinterpret_cast<const uint32_t*>(from + 2 * D), a, b);
                            }
                        }
                    }
                } else {
                    if (!wait(&ctl->op_empty[stage], op_parity)) break;
                    // drafted tokens: 16 bytes of a row at a time, neighbouring threads at neighbouring ones; values' rows behind them are zeros
                    const bool wide = f.odd & TA_WIDE;
                    const unsigned long long big = wide ? ctl->big[u % TA_UNITS] : 0;
                    const uint16_t* rows = which ? x.V + (long long)un.token0 * x.v_stride + un.head * D : x.K + (long long)un.token0 * x.k_stride + un.head * D;
                    const long long stride = which ? x.v_stride : x.k_stride;
                    constexpr int CH = D / 8;
#pragma unroll 1
                    for (int i = token; i < un.n * CH; i += TA_TILE) {
                        const int t = i / CH, c = i % CH;
                        const uint4 raw = *reinterpret_cast<const uint4*>(rows + t * stride + c * 8);
                        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
                        uint8_t* line = to + t * 128;
                        const float k0 = times_pow2(1.f, -(wide && !which ? key_exponent(ctl->draft_top[u % TA_UNITS][t], e) : e));
                        if (which == 0) {                                              // elements (0, 4, 1, 5, ..) of the chunk
                            uint32_t h[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const uint32_t u = w[k >> 1], v = w[2 + (k >> 1)];
                                h[k] = pack_f16((k & 1 ? bf16_hi(u) : bf16_lo(u)) * k0, (k & 1 ? bf16_hi(v) : bf16_lo(v)) * k0);
                            }
                            *reinterpret_cast<uint4*>(line + (c >> 3) * (TA_TILE * 128) + (((c ^ t) & 7) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
                        } else {
                            // element 16 i' + 8 j' + g is place 2 (i' mod 4) + i' / 4 of chunk 2 g + j', D = 64: place 2 i' + j' of chunk g
                            const int place = D == 128 ? 2 * ((c >> 1) & 3) + (c >> 3) : 2 * (c >> 1) + (c & 1);
#pragma unroll
                            for (int g = 0; g < 8; ++g) {
                                const float v = (g & 1 ? bf16_hi(w[g >> 1]) : bf16_lo(w[g >> 1])) * k0;
                                const int chunk = D == 128 ? 2 * g + (c & 1) : g;
                                // (what is not finite, or far larger than the rest, is put back at the end, for the rows that see it)
                                *reinterpret_cast<uint16_t*>(line + (chunk >> 3) * (TA_TILE * 128) + (((chunk ^ t) & 7) << 4) + 2 * place) =
                                    (uint16_t)pack_f16(fabsf(v) < INFINITY && !(big >> t & 1) ? v : 0.f, 0.f);
                            }
                        }
                    }
#pragma unroll 1
                    for (int i = un.n * 8 + token; i < TA_TILE * 8 && which; i += TA_TILE) {
                        *reinterpret_cast<uint4*>(to + i * 16) = make_uint4(0, 0, 0, 0);
                        if (D == 128) *reinterpret_cast<uint4*>(to + TA_TILE * 128 + i * 16) = make_uint4(0, 0, 0, 0);
                    }
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (elect_one()) {
                    mbar_arrive(smem_u32(&ctl->op_full[stage]));
                    mbar_arrive(smem_u32(&ctl->scales_empty[n % TA_SCALES]));
                    if (coded) mbar_arrive(smem_u32(&ctl->codes_empty[code_stage]));
                }
                __syncwarp();
            }
            if (!ok) break;
            n_op += 2 * nt;
            n_code += nt - drafts;
            n_tile += nt;
            leave_unit(u);
        }
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(TA_REGS_SOFT));
        // ------------------------------------------------ softmax and epilogue: thread = lane of tile w
        const int w = warp >> 2, quarter = warp & 3, r = quarter * 32 + lane;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const uint32_t t_s = tmem + lanes + w * TA_TILE, t_o = tmem + lanes + 256 + w * D;
        uint32_t n_s = 0, n_tile = 0, n_together = 0;      // score tiles of this slot so far; tiles so far
        auto together = [&]() -> bool {            // a barrier of the softmax warps, with the limit of every wait
            __syncwarp();
            if (elect_one()) mbar_arrive(smem_u32(&ctl->together));
            return wait(&ctl->together, n_together++ & 1);
        };
#pragma unroll 1
        for (uint32_t u = 0; next_unit(u); ++u) {
            const TreeUnit& un = ctl->unit[u % TA_UNITS];
            const int t0 = un.tile0, nt = un.tile1 - t0, step = un.two ? 1 : 2, j0 = un.two ? 0 : w;
            const int copies = un.copies, distinct = TA_TILE >> copies, copy = r >> (7 - copies), row = (un.two ? w * TA_TILE : 0) + (r & (distinct - 1));   // row of the unit
            const bool live = row < un.rows;
            const int buf = un.two ? w : un.buf;
            float m = -INFINITY, l = 0.f, rs = 0.f;
            int ev = 0, odd = 0;
#pragma unroll 1
            for (int j = j0; j < nt; j += step, ++n_s) {
                if (!wait(&ctl->s_full[w], n_s & 1)) break;
                tc_fence_after();
                const TreeInfo f = ctl->info[(n_tile + j) % TA_INFO];
                const bool drafts = t0 + j == 0;
                if (j == j0) rs = ctl->row_scale[buf][r & (distinct - 1)];
                const bool wide = drafts && (f.odd & TA_WIDE);
                const float c = fminf(fmaxf(times_pow2(rs, f.ek), 1e-37f), 3e38f);    // (not 0 or infinite: scores at -inf, scores of 0)
                if (wide) {                                                    // scores from their keys' exponents to the tile's
                    const uint32_t* tops = ctl->draft_top[u % TA_UNITS];
#pragma unroll 1
                    for (int b = 0; b < 4; ++b) {
                        uint32_t v[16];
                        tmem_ld_32x16(t_s + b * 16, v);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int e = key_exponent(tops[b * 16 + i], f.ek) - f.ek;
                            v[i] = __float_as_uint(__uint_as_float(v[i]) * pow2i(e >> 1) * pow2i(e - (e >> 1)));
                        }
                        tmem_st_32x16(t_s + b * 16, v);
                    }
                    tmem_st_wait();
                }
                if (drafts || f.v0 < 64 || f.v1 < 64) {
                    // what is not seen: -inf, written over the scores (the drafted tokens, a row's last tile)
                    unsigned long long see[2] = {f.v0 >= 64 ? ~0ull : (1ull << f.v0) - 1, f.v1 >= 64 ? ~0ull : (1ull << f.v1) - 1};
                    if (drafts) {
                        odd = f.odd & TA_ODD;
                        see[0] = live ? ctl->sees[buf][token_of(x, un.row0 + row)] : 0ull;
                    }
#pragma unroll 1
                    for (int b = 0; b < 4; ++b) {
                        uint32_t v[32];
                        tmem_ld_32x32(t_s + b * 32, v);
                        tmem_ld_wait();
                        const uint32_t bits = (uint32_t)((b & 2 ? see[1] : see[0]) >> (32 * (b & 1)));
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (!(bits >> i & 1)) v[i] = 0xff800000u;
                        tmem_st_32x32(t_s + b * 32, v);
                    }
                    tmem_st_wait();
                }
                // This copy's blocks of 32 keys, one after the other: where a row's maximum has grown too far beyond the reference (or V's exponent has), what there is follows.
                const int blocks = 4 >> copies, b0 = copy * blocks;
                const f32x2 c2 = pack2(c, c);
                f32x2 sum = pack2(0.f, 0.f);
                if (j == j0) ev = f.ev;
#pragma unroll 1
                for (int b = b0; b < b0 + blocks; ++b) {
                    uint32_t v[32];
                    tmem_ld_32x32(t_s + 32 * b, v);
                    tmem_ld_wait();
                    float t0 = -INFINITY, t1 = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        t0 = max3(t0, __uint_as_float(v[i]), __uint_as_float(v[i + 1]));
                        t1 = max3(t1, __uint_as_float(v[i + 2]), __uint_as_float(v[i + 3]));
                    }
                    const float top = fmaxf(t0, t1) * c;
                    const bool grow = top > m && !(top - m <= TA_LAZY);
                    if (__any_sync(0xffffffffu, grow) || ev != f.ev) {
                        const float to = floorf(top), g = !grow ? 1.f : m - to < -126.f ? 0.f : pow2i((int)(m - to));
                        if (grow) m = to;
                        l *= g;
                        sum = mul2(sum, pack2(g, g));
                        if (j != j0) {                                         // the outputs, once the last product has landed
                            if (!wait(&ctl->pv_done[w], (n_s - 1) & 1)) break;
                            tc_fence_after();
                            const float go = ev == f.ev ? g : ev - f.ev < -126 ? 0.f : g * pow2i(min(ev - f.ev, 127));
#pragma unroll 1
                            for (int d = 0; d < D; d += 16) {
                                uint32_t ov[16];
                                tmem_ld_32x16(t_o + d, ov);
                                tmem_ld_wait();
#pragma unroll
                                for (int i = 0; i < 16; ++i) ov[i] = __float_as_uint(__uint_as_float(ov[i]) * go);
                                tmem_st_32x16(t_o + d, ov);
                            }
                        }
                        ev = f.ev;
                        // this tile's probabilities so far: times 2^-24 at the least (fp16 has no smaller power), and what is left of g before that, whose rounding the 2^-24 makes small
                        const float g1 = fmaxf(g, 0x1p-24f), g0 = g >= 0x1p-24f ? 1.f : g * 0x1p24f;
                        const uint32_t g12 = pack_f16(g1, g1), g02 = pack_f16(g0, g0);
#pragma unroll 1
                        for (int e = b0; e < b; ++e) {
                            uint32_t q[16];
                            tmem_st_wait();
                            tmem_ld_32x16(t_s + 64 * (e >> 1) + 16 * (e & 1), q);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 16; ++i) q[i] = mul_f16x2(mul_f16x2(q[i], g02), g12);
                            tmem_st_32x16(t_s + 64 * (e >> 1) + 16 * (e & 1), q);
                        }
                        tmem_st_wait();
                    }
                    const float ref = (m == -INFINITY ? 0.f : -m) + TA_SHIFT;
                    const f32x2 ref2 = pack2(ref, ref);
                    uint32_t p[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float x0, x1;
                        unpack2(fma2(pack2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), c2, ref2), x0, x1);
                        x0 = ex2_ftz(x0);
                        x1 = ex2_ftz(x1);
                        sum = add2(sum, pack2(x0, x1));
                        p[i] = pack_f16(x0, x1);
                    }
                    tmem_st_32x16(t_s + 64 * (b >> 1) + 16 * (b & 1), p);      // (over scores that have been read: block 0's lie there, or block 2's)
                }
                if (!ok) break;
                if (copies) {
                    uint32_t zero[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) zero[i] = 0;
#pragma unroll 1
                    for (int b = 0; b < 4; ++b)
                        if ((b >> (2 - copies)) != copy) tmem_st_32x16(t_s + 64 * (b >> 1) + 16 * (b & 1), zero);
                }
                float sum0, sum1;
                unpack2(sum, sum0, sum1);
                l += sum0 + sum1;
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (elect_one()) mbar_arrive(smem_u32(&ctl->p_full[w]));
            }
            if (!ok) break;
            n_tile += nt;
            const bool have = j0 < nt;
            if (have) {
                if (!wait(&ctl->pv_done[w], (n_s - 1) & 1)) break;
                tc_fence_after();
            }
            // ---- the end of the unit, or of this block's share of it.  What the copies of a row have becomes one: a warp reads both slots' outputs of its lanes, group w of warps
            // the columns of rounds 2 w and 2 w + 1 (with more than 128 rows: its own slot's, all of them); copies in other lanes follow by way of shared memory.
            constexpr int CW = D / 4, CQ = CW / 4;                             // columns of a round: elements 16 i .. 16 i + 15 and, D = 128, 64 + 16 i .. + 15; in fours
            const bool two = un.two, to_part = un.slot >= 0;
            float2* stats = &ctl->stats[w * TA_TILE + r];
            *stats = make_float2(m, have ? l : 0.f);
            if (lane == 0) ctl->ev[warp] = ev;
            if (warp == 0 && lane == 0) ctl->odd = odd;
            tc_fence_before();
            if (!together()) break;
            tc_fence_after();
            float ref, all = 0.f;
            {
                // the row's 1, 2, 4 or 8 parts, `distinct` lanes apart: each is read 8, 4, 2 or 1 times, by all lanes of the row in the same order
                const int apart = two ? 0 : distinct, at0 = two ? w * TA_TILE + r : r & (distinct - 1);
                float2 part[8];
                float top = -INFINITY;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    part[k] = ctl->stats[(at0 + k * apart) & (2 * TA_TILE - 1)];
                    top = fmaxf(top, part[k].x);
                }
                ref = top == -INFINITY ? 0.f : top;
#pragma unroll
                for (int k = 0; k < 8; ++k) all += part[k].y == 0.f ? 0.f : part[k].y * ex2_ftz(part[k].x - ref);
                all *= two ? 0.125f : 0.25f * (1 << copies);
            }
            ctl->sums[w * TA_TILE + r] = make_float2(ref, all);
            if (to_part && live) x.stats[(size_t)un.slot * x.part_rows + row] = make_float2(ref, all);    // (the copies of a row write the same)
            // factors of what this lane has in slot 0 (its own slot) and in slot 1; 0: what stands there does not count
            const int va = two ? w : 0;
            const bool second = !two && nt > 1;
            auto factor = [&](int v) -> float {
                const float2 st = ctl->stats[v * TA_TILE + r];
                return st.y != 0.f && all != 0.f ? ex2_ftz(st.x - ref) / all : 0.f;
            };
            const float fa = factor(va), fb = second ? factor(1) : 0.f;
            const int ea = ctl->ev[va * 4 + quarter], eb = ctl->ev[4 + quarter];
            const float a1 = fa * pow2i(ea >> 1), a2 = pow2i(ea - (ea >> 1)), b1 = fb * pow2i(eb >> 1), b2 = pow2i(eb - (eb >> 1));
            float4* stage = reinterpret_cast<float4*>(q_smem + un.buf * C::op_bytes);        // the unit's Q has been used up
            const bool any_odd = ctl->odd != 0, direct = copies == 0 && !any_odd;
            const int items = un.rows * CQ, own_at = un.row0 + row, own_token = token_of(x, own_at);
            float* own_part = x.part + ((size_t)max(un.slot, 0) * x.part_rows + row) * D;
            uint16_t* own_out = x.O + (long long)(un.token0 + own_token) * x.o_stride + (un.head * x.G + own_at - own_token * x.G) * D;
#pragma unroll 1
            for (int i = two ? 0 : 2 * w; i < (two ? 4 : 2 * w + 2); ++i) {
                // four elements at a time, 4 q of the round's first 16 and (D = 128) of the other 16, or of its first and last 8 (a loop: this code runs once a unit, and most of its
                // time is the fetching of instructions)
#pragma unroll 1
                for (int q = 0; q < CQ / 2; ++q) {
                    const uint32_t from = tmem + lanes + 256 + va * D + 2 * i + (D == 128 ? ((q & 1) * 8 + (q >> 1)) * 8 : q * 32), also = second ? from + D : from;
                    uint32_t y[8], z[8];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        tmem_ld_32x2(from + k * (D == 128 ? 16 : 8), y[k], y[4 + k]);
                        tmem_ld_32x2(also + k * (D == 128 ? 16 : 8), z[k], z[4 + k]);
                    }
                    tmem_ld_wait();
                    float o[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float ya = __uint_as_float(y[k]) * a1 * a2, zb = __uint_as_float(z[k]) * b1 * b2;
                        o[k] = (fa != 0.f ? ya : 0.f) + (fb != 0.f ? zb : 0.f);
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float4 v = make_float4(o[4 * h], o[4 * h + 1], o[4 * h + 2], o[4 * h + 3]);
                        const int k = q + h * (CQ / 2), d0 = (D == 128 ? 64 * h : 8 * h) + 16 * i + 4 * q;
                        if (!direct) stage[(w * TA_TILE + r) * CQ + (k ^ (lane & (CQ - 1)))] = v;
                        else if (live && to_part) *reinterpret_cast<float4*>(own_part + d0) = v;           // (a lane has its row to itself)
                        else if (live) *reinterpret_cast<uint2*>(own_out + d0) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
                    }
                    __syncwarp();
                }
                if (direct) continue;
                if (!together()) break;
                // four elements of a row: of both halves of the warps' rounds, or of both halves of the rows
#pragma unroll 1
                for (int item = tid; item < (two ? items : 2 * items); item += TA_SOFT * 32) {
                    const int half = two ? 0 : item >= items, to_row = (item - half * items) / CQ, k0 = (item - half * items) % CQ;
                    const int d0 = (D == 128 && k0 >= 4 ? 48 : 0) + 16 * (two ? i : 2 * half + (i & 1)) + 4 * k0;
                    const float4* from = stage + (half * TA_TILE + to_row) * CQ + (k0 ^ (to_row & (CQ - 1)));      // (the copies' lanes: the same swizzle)
                    float4 v = *from;
#pragma unroll 1
                    for (int p = 1; p < 1 << copies; ++p) {
                        from += distinct * CQ;
                        const float4 y = *from;
                        v.x += y.x;
                        v.y += y.y;
                        v.z += y.z;
                        v.w += y.w;
                    }
                    const int at = un.row0 + to_row, token = token_of(x, at);
                    if (any_odd) {                                             // what the row sees of drafted values that are not in the products
                        const unsigned long long sees = ctl->sees[un.buf][token], big = ctl->big[u % TA_UNITS];
                        const uint16_t* q = x.Q + (long long)(un.token0 + token) * x.q_stride + (un.head * x.G + at - token * x.G) * D;
#pragma unroll 1
                        for (int t = 0; t < un.n; ++t) {
                            if (!(sees >> t & 1)) continue;
                            float p = 0.f;
                            if (big >> t & 1) {
                                const uint16_t* key = x.K + (un.token0 + (long long)t) * x.k_stride + un.head * D;
                                float dot = 0.f;
#pragma unroll 1
                                for (int d = 0; d < D; ++d) dot = fmaf(__uint_as_float((uint32_t)q[d] << 16), __uint_as_float((uint32_t)key[d] << 16), dot);
                                const float2 of = ctl->sums[to_row];
                                p = ex2_ftz(dot * x.scale_log2e - of.x + TA_SHIFT) / of.y;
                            }
                            const uint2 y = *reinterpret_cast<const uint2*>(x.V + (un.token0 + (long long)t) * x.v_stride + un.head * D + d0);
                            v.x += left_out(p, bf16_lo(y.x));
                            v.y += left_out(p, bf16_hi(y.x));
                            v.z += left_out(p, bf16_lo(y.y));
                            v.w += left_out(p, bf16_hi(y.y));
                        }
                    }
                    if (to_part)
                        *reinterpret_cast<float4*>(x.part + ((size_t)un.slot * x.part_rows + to_row) * D + d0) = v;
                    else
                        *reinterpret_cast<uint2*>(x.O + (long long)(un.token0 + token) * x.o_stride + (un.head * x.G + at - token * x.G) * D + d0) =
                            make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
                }
                if (!together()) break;
            }
            if (!ok || (direct && !together())) break;         // (the outputs of either slot and the statistics have been read)
            if (!ok) break;
            tc_fence_before();
            __syncwarp();
            if (lane == 0)
                for (int b = 0; b < 2; ++b)
                    if (un.two || un.buf == b) mbar_arrive(smem_u32(&ctl->q_empty[b]));
            leave_unit(u);
        }
        if (!ok) tmem_st_wait();
        tc_fence_before();
    }
    if (!ok) ctl->abort_flag = 1;
    __syncthreads();
    if (ctl->abort_flag) {
        // a role gave up: what the others have issued (products, copies into shared memory) may be in flight still, and is waited for, bounded as well, before the block leaves
        if (warp == 8 && elect_one()) {
            tc_commit(smem_u32(&ctl->drain));
            int dummy = 0;
            mbar_wait(smem_u32(&ctl->drain), 0, &dummy, 2000000ull);
        }
        if (tid == 0) {
            const uint64_t t0 = globaltimer_ns();
            while (globaltimer_ns() - t0 < 2000000ull) __nanosleep(1000);
            *x.status = AG_ERR_TIMEOUT;
        }
        __syncthreads();
    }
    if (warp == 8) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// Units that several blocks share: O = sum_c w_c O_c / sum_c w_c, w_c = 2^(m_c - m) l_c.  Column i of the grid joins the unit that began in block i of the main kernel and
// went on beyond it, a warp for each of its rows: the lanes weigh the parts side by side, then each adds up its elements of all of them.
constexpr int TJ_WARPS = 8;
template <int D>
__global__ void __launch_bounds__(TJ_WARPS * 32) k_attn_tree_join(const TreeArgs x, int blocks) {
    constexpr int E = D / 32;                      // elements of a lane
    __shared__ float weight[TJ_WARPS][TA_BLOCKS];
    __shared__ int slot[TJ_WARPS][TA_BLOCKS];
    dep_wait();
    const TreeCross c = x.cross[blockIdx.x];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.y * TJ_WARPS + warp;
    if (row >= c.rows) return;
    // blocks from this one on, while they have tiles of the unit
    const int last = (int)min((long long)blocks - 1, (c.begin + c.unit_places + (long long)c.weight * c.tiles - 1) / c.quota), n = last - (int)blockIdx.x + 1;
    float top = -INFINITY;
#pragma unroll 1
    for (int i = lane; i < n; i += 32) {
        const int b = blockIdx.x + i;
        const int t0 = tiles_before(c.quota * b, c.begin, c.unit_places, c.weight, c.tiles), t1 = tiles_before(c.quota * (b + 1), c.begin, c.unit_places, c.weight, c.tiles);
        const int at = 2 * b + (t1 < c.tiles ? 1 : 0);
        slot[warp][i] = t0 < t1 ? at : -1;
        const float2 s = t0 < t1 ? __ldcg(&x.stats[(size_t)at * x.part_rows + row]) : make_float2(-INFINITY, 0.f);
        weight[warp][i] = s.y;
        if (s.y != 0.f) top = fmaxf(top, s.x);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
#pragma unroll 1
    for (int i = lane; i < n; i += 32) {
        const float l = weight[warp][i];
        const float f = l == 0.f ? 0.f : l * ex2_ftz(__ldcg(&x.stats[(size_t)slot[warp][i] * x.part_rows + row]).x - ref);
        weight[warp][i] = f;
        sum += f;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    __syncwarp();
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    float v[E];
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = 0.f;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
        const int at = slot[warp][i];
        if (at < 0) continue;
        const float f = weight[warp][i] * inv;
        const float* from = x.part + ((size_t)at * x.part_rows + row) * D + lane * E;
        float u[E];
        if constexpr (E == 4) {
            const float4 q = __ldcg(reinterpret_cast<const float4*>(from));
            u[0] = q.x; u[1] = q.y; u[E - 2] = q.z; u[E - 1] = q.w;
        } else {
            const float2 q = __ldcg(reinterpret_cast<const float2*>(from));
            u[0] = q.x; u[1] = q.y;
        }
#pragma unroll
        for (int k = 0; k < E; ++k) v[k] += f == 0.f && fabsf(u[k]) < INFINITY ? 0.f : f * u[k];
    }
    const int at = c.row0 + row, token = token_of(x, at);
    uint16_t* out = x.O + (long long)(c.token0 + token) * x.o_stride + (c.head * x.G + at - token * x.G) * D + lane * E;
#pragma unroll
    for (int k = 0; k < E; k += 2) *reinterpret_cast<uint32_t*>(out + k) = pack_bf16(v[k], v[k + 1]);
}

static bool tree_shape_ok(long long n_seq, int max_tokens, int H_q, int H_kv, int D, int max_pages) {
    return n_seq >= 1 && max_tokens >= 1 && max_tokens <= AG_TREE_MAX && H_kv >= 1 && H_kv <= 1024 && H_q >= H_kv && H_q % H_kv == 0 && H_q / H_kv <= 64 &&
           (D == 64 || D == 128) && max_pages >= 1 && max_pages < (1 << 25);
}
static int tree_part_rows(int max_tokens, int G) { return std::min(256, max_tokens * G); }
static size_t round256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace ag

using namespace ag;

extern "C" size_t ag_attention_tree_kv4_workspace(int n_seq, int max_tokens, int H_q, int H_kv, int D, int max_pages) {
    if (!tree_shape_ok(n_seq, max_tokens, H_q, H_kv, D, max_pages)) return 0;
    const size_t rows = (size_t)tree_part_rows(max_tokens, H_q / H_kv);
    return 256 + round256(TA_BLOCKS * sizeof(TreeCross)) + round256(2 * TA_BLOCKS * rows * sizeof(float2)) + 2 * TA_BLOCKS * rows * D * sizeof(float);
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
    constexpr int smem128 = TCfg<128>::smem_bytes, smem64 = TCfg<64>::smem_bytes > TA_MIN_SMEM ? TCfg<64>::smem_bytes : TA_MIN_SMEM;
    static std::atomic<unsigned long long> attr_done{0};
    const cudaError_t attr_err = once_per_device(attr_done, [] {
        cudaError_t e = cudaFuncSetAttribute(k_attn_tree_kv4<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem128);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k_attn_tree_kv4<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem64);
        // the softmax warps ask for registers out of those that the block is launched with: fewer would be waited for without end
        for (const void* k : {(const void*)k_attn_tree_kv4<128>, (const void*)k_attn_tree_kv4<64>}) {
            cudaFuncAttributes fa;
            if (e == cudaSuccess) e = cudaFuncGetAttributes(&fa, k);
            if (e == cudaSuccess && fa.numRegs * TA_THREADS < TA_SOFT * 32 * TA_REGS_SOFT + (TA_THREADS - TA_SOFT * 32) * TA_REGS_OTHER) e = cudaErrorInvalidConfiguration;
        }
        return e;
    });
    if (attr_err != cudaSuccess) return cuda_fail(attr_err);
    TreeArgs x;
    memset(&x, 0, sizeof x);
    x.Q = (const uint16_t*)a->Q; x.K = (const uint16_t*)a->K; x.V = (const uint16_t*)a->V; x.O = (uint16_t*)a->O;
    x.pages = (const uint8_t*)pool->pages;
    x.q_stride = a->q_stride; x.k_stride = a->k_stride; x.v_stride = a->v_stride; x.o_stride = a->o_stride; x.n_tokens = (int)a->n_tokens;
    x.row = a->row; x.off = a->off; x.parent = a->parent; x.page_of = table->page_of; x.len = table->len;
    x.H_q = a->H_q; x.H_kv = H_kv; x.G = a->H_q / H_kv; x.n_seq = a->n_seq; x.n_rows = table->n_rows; x.max_pages = table->max_pages; x.n_pages = (int)pool->n_pages;
    x.max_tokens = a->max_tokens;
    x.most_len = (int)std::min<long long>(64ll * table->max_pages, 0x7fffffff);
    x.by_g = x.G > 1 ? (uint32_t)((0x100000000ull + x.G - 1) / x.G) : 0;
    x.part_rows = tree_part_rows(a->max_tokens, x.G);
    x.scale_log2e = 1.4426950408889634f * (a->scale > 0.f ? a->scale : 1.f / sqrtf((float)D));
    uint8_t* ws = (uint8_t*)workspace;
    x.status = (int32_t*)ws;
    x.cross = (TreeCross*)(ws + 256);
    x.stats = (float2*)((uint8_t*)x.cross + round256(TA_BLOCKS * sizeof(TreeCross)));
    x.part = (float*)((uint8_t*)x.stats + round256(2 * TA_BLOCKS * (size_t)x.part_rows * sizeof(float2)));
    // no more blocks than there can be tiles
    const long long unit_weight = (a->max_tokens * x.G + 127) / 128, most = (long long)a->n_seq * H_kv * unit_weight * ((table->max_pages + 1) / 2 + 1);
    const int blocks = (int)std::min<long long>(TA_BLOCKS, most);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(TA_THREADS);
    cfg.dynamicSmemBytes = D == 128 ? smem128 : smem64;
    cfg.stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    AG_CUDA(cudaLaunchKernelEx(&cfg, D == 128 ? k_attn_tree_kv4<128> : k_attn_tree_kv4<64>, x));
    count_launch();
    cfg.gridDim = dim3((unsigned)blocks, (unsigned)((x.part_rows + TJ_WARPS - 1) / TJ_WARPS));
    cfg.blockDim = dim3(TJ_WARPS * 32);
    cfg.dynamicSmemBytes = 0;
    AG_CUDA(cudaLaunchKernelEx(&cfg, D == 128 ? k_attn_tree_join<128> : k_attn_tree_join<64>, x, blocks));
    count_launch();
    return AG_OK;
}
