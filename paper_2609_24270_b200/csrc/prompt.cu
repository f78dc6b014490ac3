// Attention over whole prompts: causal or not, grouped query heads, packed sequences of different lengths, keys that may begin before the
// queries (a later chunk of a prompt).  Runs on the SMs of a plan like every persistent kernel here: one block per planned SM,
// units of work from one queue, longest first.
//
// Work unit = (sequence, KV head, 2 x 128 / G consecutive tokens), G = query heads per KV head: the rows of a tile are (token, head of the
// group) pairs, so that a tile of 128 rows spans only 128 / G tokens (little of the causal triangle's edge is wasted, a short chunk
// still fills the MMA) and all heads of a group share the key and value tiles.  Per unit two such tiles, w = 0, 1, and tiles of 128 keys:
//     S_w = Q_w K_j^T              tcgen05.mma, 128 x 128 x D, scores in tensor memory
//     P_w = 2^((S_w - m) scale log2 e)   one thread per row (128 threads per tile); P as bf16 back into tensor memory, over the scores
//     O_w += P_w V_j               tcgen05.mma with the A operand in tensor memory, 128 x D x 128, outputs in tensor memory
//     O_w / sum(P_w)               epilogue
// While the softmax of one tile runs, the tensor core works on the other: PV_0(j), S_0(j + 1), PV_1(j), S_1(j + 1), ...  The reference
// m of a row moves only when its maximum has grown by more than 8 (in log2 units): then, and only then, the outputs are rescaled.  P is
// at most 2^8, sums and outputs are in 32 bits, so this changes no rounding.
// The tensor pipe and, as closely, the exponentials: a pair of 128 x 128 tiles takes 2 x 1024 cycles of MMAs (D = 128) and 2 x 1024 cycles of the
// special-function units (16 per cycle and SM).  What bounds it is a tile's own chain, 1760 cycles of softmax and 1280 until its next scores are there;
// more tiles in flight do not fit tensor memory at D = 128 (at 64 a third score tile would; not built).  8192 tokens, 32 query heads on 8, D = 128,
// causal: 445 us, 1235 TFLOP/s (0.74 of the measured product of matrices; 520 us once the power cap holds), not causal 850; D = 64: 390 and 740.
//
// A probability of zero times a later token's infinity or NaN, in a key tile that rows share, spoils a row that does not see that token.  A causal unit
// with a result that is not finite is therefore run a second time, with the values that are not finite taken as zeros while the first of
// each kind is noted for every column: what a row sees of them decides what it adds to the row (second pass, below).  Twice the work and
// the scan of the value tiles, for such units only.
#include <string.h>

#include <algorithm>

#include "persist.cuh"

namespace ag {

constexpr int PA_M = 128;                 // rows of a tile
constexpr int PA_N = 128;                 // keys of a tile
constexpr int PA_STAGES = 4;              // K and V tiles in turn
constexpr int PA_THREADS = 384;           // warps 0-3 softmax of tile 0, 4-7 of tile 1, 8 MMA, 9 units + Q, 10 K, 11 V
constexpr int PA_MAXSEQ = 1024;           // sequences of one launch
constexpr int PA_CONSUMERS = 8 + 3;       // warps that read the unit: softmax, MMA, K, V
constexpr float PA_LAZY = 8.f;
// One pair in eight takes its exponentials from the multiply-add units (exp2_cubic): at 8192 tokens x 32 heads, D = 128, 464 us with none,
// 456 with one, 459 with two, 475 with three; D = 64: 440, 396, 449, 446 (figures of that step).
constexpr int PA_CUBIC = 1;

struct PromptArgs {
    uint16_t* O;
    const uint16_t *Q, *K, *V;
    const int32_t *q_off, *kv_off;        // [n_seq + 1]
    long long q_stride, k_stride, v_stride, o_stride, q_tokens, kv_tokens;
    int H_q, H_kv, G, tpt, n_seq, causal; // tpt: tokens of a tile
    float scale_log2e;
};

struct PromptSeq {                        // a sequence in the order of work
    int q0, q_len, k0, k_len;
};

struct PromptCtl {
    uint64_t q_full[2], q_empty[2];
    uint64_t kv_full[PA_STAGES], kv_empty[PA_STAGES];
    uint64_t s_full[2], p_full[2], pv_done[2];
    uint64_t unit_full, unit_empty;
    uint64_t tail, mma_drain, scanned[2];
    int unit[4];                          // sequence (in order of work; -1: the end), KV head, first token, 1: second pass
    uint32_t spoilt[4];                   // k + 1 in place k mod 4: the k-th unit had a result that is not finite
    int first_odd[2][3][128];             // second pass, units in turn: the first key with a NaN, an infinity, a negative one in the column
    uint32_t tmem_base;
    int abort_flag, member, slot;
    int blocks_before[PA_MAXSEQ + 1];     // units of one head in front of the i-th sequence of work
    PromptSeq seq[PA_MAXSEQ];
};

template <int D>
struct PCfg {
    static constexpr int q_bytes = PA_M * D * 2;
    static constexpr int kv_bytes = PA_N * D * 2;
    static constexpr int smem_bytes = 2 * q_bytes + PA_STAGES * kv_bytes + (int)((sizeof(PromptCtl) + 1023) / 1024 * 1024) + 1024;
};
static_assert(PCfg<128>::smem_bytes <= 227 * 1024, "does not fit");
// one block per SM, whatever else the tile size would allow: the plan counts on it, and the block takes all of the SM's tensor memory
constexpr int PA_MIN_SMEM = 200 * 1024;

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// 2^x on the multiply-add units: x = n + f with n the nearest integer, 2^f by the cubic with the smallest largest relative error on
// [-1/2, 1/2] (7.5e-5, from an exchange algorithm; bf16 rounds at 2e-3), 2^n through the exponent field, which is 0 for
// n = -127: what is below 2^-126.5, a masked key's -inf among it, gives exactly 0.  NaN stays NaN.
__device__ __forceinline__ f32x2 exp2_cubic(f32x2 v) {
    float v0, v1, t0, t1;
    unpack2(v, v0, v1);
    const f32x2 x = pack2(max_nan(v0, -127.f), max_nan(v1, -127.f));
    constexpr float M = 12582912.f + 127.f;                // 1.5 * 2^23: the sum's low bits are n + 127
    const f32x2 t = add2(x, pack2(M, M));
    const f32x2 f = fma2(add2(t, pack2(-M, -M)), pack2(-1.f, -1.f), x);
    f32x2 q = fma2(f, pack2(0.05517167f, 0.05517167f), pack2(0.24261112f, 0.24261112f));
    q = fma2(q, f, pack2(0.69326099f, 0.69326099f));
    q = fma2(q, f, pack2(0.99992807f, 0.99992807f));
    unpack2(t, t0, t1);
    return mul2(q, pack2(__uint_as_float(__float_as_uint(t0) << 23), __uint_as_float(__float_as_uint(t1) << 23)));
}
// 32 bytes: in one store where the address allows (lanes are rows apart, and the other warps' barriers queue behind such stores: 4 units of one
// key tile a block took 38.3 us with 16-byte stores, 35.3 with these)
__device__ __forceinline__ void store32(uint16_t* to, const uint32_t (&v)[8], bool wide) {
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
    } else {
        reinterpret_cast<uint4*>(to)[0] = make_uint4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<uint4*>(to)[1] = make_uint4(v[4], v[5], v[6], v[7]);
    }
}

// keys that token i of a sequence sees: 0 .. last_key(i); may be negative
__device__ __forceinline__ int last_key(const PromptArgs& x, const PromptSeq& s, int i) {
    return x.causal ? min(s.k_len - 1, s.k_len - s.q_len + i) : s.k_len - 1;
}
// key tiles of tile w of the unit whose first token is t0 (0: no token, or no token that sees a key)
__device__ __forceinline__ int key_tiles(const PromptArgs& x, const PromptSeq& s, int t0, int w) {
    const int first = t0 + w * x.tpt;
    if (first >= s.q_len) return 0;
    return max(0, last_key(x, s, min(first + x.tpt, s.q_len) - 1) + PA_N) / PA_N;
}

// true for every thread of the block when one of them says so; all come here the same number of times
__device__ __forceinline__ bool block_any(bool mine) {
    uint32_t r;
    asm volatile(
        "{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.or.pred q, 1, %2, p;\n selp.u32 %0, 1, 0, q;\n}"
        : "=r"(r) : "r"((uint32_t)mine), "n"(PA_THREADS) : "memory");
    return r != 0;
}

// Second pass: a landed tile of values (64-column blocks of 128 rows of 128 bytes, 16-byte pieces swizzled by the row), rows 0 .. valid - 1 are keys
// key0 .. of the sequence.  One warp, a lane keeps to eight columns: what is not finite becomes zero, the first of each kind is noted by column.
// Two elements a word: without their signs, 0x80 more makes bit 15 of what is not finite, 0x7f more that of a NaN.
template <int D>
__device__ __forceinline__ void take_out_odd(uint8_t* tile, int valid, int key0, int (*first_odd)[128]) {
    const int lane = threadIdx.x & 31, piece = lane & 7;
#pragma unroll 1
    for (int d = 0; d < D / 64; ++d) {
        uint32_t noted[3][4] = {};                 // by this lane, of this tile
#pragma unroll 1
        for (int row = lane >> 3; row < valid; row += 4) {
            uint4* at = reinterpret_cast<uint4*>(tile + d * (PA_N * 128) + row * 128 + ((piece ^ (row & 7)) << 4));
            const uint4 v = *at;
            uint32_t w[4] = {v.x, v.y, v.z, v.w}, kind[3][4], any = 0, fresh = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) any |= (w[k] & 0x7fff7fffu) + 0x00800080u;
            if (!(any & 0x80008000u)) continue;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t t = w[k] & 0x7fff7fffu, bad = (t + 0x00800080u) & 0x80008000u;
                kind[0][k] = (t + 0x007f007fu) & 0x80008000u;
                kind[1][k] = (bad ^ kind[0][k]) & ~w[k];
                kind[2][k] = (bad ^ kind[0][k]) & w[k];
                w[k] &= ~((bad >> 15) * 0xffffu);
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    kind[i][k] &= ~noted[i][k];
                    noted[i][k] |= kind[i][k];
                    fresh |= kind[i][k];
                }
            }
            if (fresh) {
#pragma unroll
                for (int i = 0; i < 3; ++i)
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (kind[i][k >> 1] & (k & 1 ? 0x80000000u : 0x8000u)) atomicMin(&first_odd[i][d * 64 + piece * 8 + k], key0 + row);
            }
            *at = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

template <int D>
__global__ void __launch_bounds__(PA_THREADS, 1)
k_attn_prompt(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
              const PersistParams p, const PromptArgs x) {
    using C = PCfg<D>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base - raw);
    const uint32_t q_base = base, kv_base = base + 2 * C::q_bytes;
    PromptCtl* ctl = reinterpret_cast<PromptCtl*>(smem + 2 * C::q_bytes + PA_STAGES * C::kv_bytes);
    volatile int* abort_flag = &ctl->abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 32) {
        ctl->abort_flag = 0;
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&ctl->q_full[i]), 1);
            mbar_init(smem_u32(&ctl->q_empty[i]), 1);
            mbar_init(smem_u32(&ctl->s_full[i]), 1);
            mbar_init(smem_u32(&ctl->p_full[i]), 4);
            mbar_init(smem_u32(&ctl->pv_done[i]), 1);
        }
        for (int i = 0; i < PA_STAGES; ++i) {
            mbar_init(smem_u32(&ctl->kv_full[i]), 1);
            mbar_init(smem_u32(&ctl->kv_empty[i]), 1);
        }
        mbar_init(smem_u32(&ctl->unit_full), 1);
        mbar_init(smem_u32(&ctl->unit_empty), PA_CONSUMERS);
        for (int i = 0; i < 4; ++i) ctl->spoilt[i] = 0xffffffffu;
        for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&ctl->scanned[i]), 1);
        mbar_init(smem_u32(&ctl->tail), 1);
        mbar_init(smem_u32(&ctl->mma_drain), 1);
        mbar_fence_init();
        prefetch_tmap(&tm_q);
        prefetch_tmap(&tm_k);
        prefetch_tmap(&tm_v);
    } else if (tid == 64) {
        // join the plan: the slot of this block's SM, unless another block has it
        const int slot = p.quick[smid()].x;
        ctl->slot = slot;
        ctl->member = slot >= 0 && atomicMax(&p.claimed[slot], p.epoch) < p.epoch;
    }
    // ---- order of work: sequences by falling number of keys (ties in the given order), each from its last tokens to its first, so that
    // long units come first and short ones fill the end.  Up to 32 sequences are put in order by one warp while the others set up.
    const int block_tokens = 2 * x.tpt;
    auto seq_at = [&](int i) {
        // offsets are clamped: whatever they hold, nothing outside the tensors is read as a sequence
        const int q0 = (int)min(max((long long)x.q_off[i], 0ll), x.q_tokens), q1 = (int)min((long long)x.q_off[i + 1], x.q_tokens);
        const int k0 = (int)min(max((long long)x.kv_off[i], 0ll), x.kv_tokens), k1 = (int)min((long long)x.kv_off[i + 1], x.kv_tokens);
        return PromptSeq{q0, max(0, q1 - q0), k0, max(0, k1 - k0)};
    };
    const bool few = x.n_seq <= 32;
    if (few) {
        if (warp == 0) {
            PromptSeq mine{0, 0, 0, -1};
            if (lane < x.n_seq) mine = seq_at(lane);
            int rank = 0;
            for (int j = 0; j < x.n_seq; ++j) {
                const int other = __shfl_sync(0xffffffffu, mine.k_len, j);
                rank += other > mine.k_len || (other == mine.k_len && j < lane);
            }
            if (lane < x.n_seq) ctl->seq[rank] = mine;
        }
    } else {
        for (int i = tid; i < x.n_seq; i += PA_THREADS) ctl->seq[i] = seq_at(i);
    }
    __syncthreads();
    if (!ctl->member) {
        if (ctl->slot < 0) wait_until_manned(p);
        return;
    }
    if (!few) {
        int rank[(PA_MAXSEQ + PA_THREADS - 1) / PA_THREADS];
        PromptSeq mine[(PA_MAXSEQ + PA_THREADS - 1) / PA_THREADS];
#pragma unroll
        for (int k = 0; k < (PA_MAXSEQ + PA_THREADS - 1) / PA_THREADS; ++k) {
            const int i = tid + k * PA_THREADS;
            rank[k] = -1;
            if (i < x.n_seq) {
                mine[k] = ctl->seq[i];
                rank[k] = 0;
                for (int j = 0; j < x.n_seq; ++j) rank[k] += ctl->seq[j].k_len > mine[k].k_len || (ctl->seq[j].k_len == mine[k].k_len && j < i);
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < (PA_MAXSEQ + PA_THREADS - 1) / PA_THREADS; ++k)
            if (rank[k] >= 0) ctl->seq[rank[k]] = mine[k];
        __syncthreads();
    }
    if (warp == 0) {
        const long long most = 0x7fffffff / x.H_kv;   // units are counted in 31 bits; only sequences that lie over one another could need more
        long long sum = 0;
        for (int i0 = 0; i0 < x.n_seq; i0 += 32) {
            const int i = i0 + lane;
            const int v = i < x.n_seq ? (ctl->seq[i].q_len + block_tokens - 1) / block_tokens : 0;
            long long inc = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long u = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += u;
            }
            if (i < x.n_seq) ctl->blocks_before[i] = (int)min(sum + inc - v, most);
            sum += __shfl_sync(0xffffffffu, inc, 31);
        }
        if (lane == 0) ctl->blocks_before[x.n_seq] = (int)min(sum, most);
    }
    if (warp == 8) {
        tmem_alloc(smem_u32(&ctl->tmem_base), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctl->tmem_base;
    const uint64_t limit = p.wait_limit_ns;
    const uint32_t idesc_s = make_idesc_bf16(PA_M, PA_N, 0, 0), idesc_o = make_idesc_bf16(PA_M, D, 0, 1);

    // the next unit: warp-uniform; false when a wait ran out.  Every consumer warp reads every unit once.
    auto next_unit = [&](uint32_t it, int& seq, int& head, int& t0, int& second) -> bool {
        if (!mbar_wait_all(smem_u32(&ctl->unit_full), it & 1, abort_flag, limit)) {
            if (lane == 0) report_timeout(p, 3);
            return false;
        }
        seq = ctl->unit[0];
        head = ctl->unit[1];
        t0 = ctl->unit[2];
        second = ctl->unit[3];
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->unit_empty));
        return true;
    };

    // After the end (unit `it`) every warp comes here, and on unless the unit in front of it has to be run once more.  A warp that gave up comes
    // here too, once, and ends it for all.
    bool over = false;
    auto all_done = [&](uint32_t it) {
        tc_fence_before();
        __syncwarp();
        over = block_any(false) || *reinterpret_cast<volatile uint32_t*>(&ctl->spoilt[(it - 1) & 3]) != it;
        return over;
    };

    // The softmax threads hold a row of 128 scores: 2 x 128 x 208 + 128 x 88 registers, as many as 384 x 168 at launch.
    if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 9) {
        // ------------------------------------------------ units, and their query rows
        // Unit i < b is the first one of the block in slot i, without asking anybody; the others come from the queue; at last the first units of
        // planned SMs that never got a block (whose slots are then taken, so that the plan counts as manned).
        const int n_units = ctl->blocks_before[x.n_seq] * x.H_kv;
        uint32_t nq[2] = {0, 0};
        int phase = 0, scan = 0, u = -1;
        bool in_hand = false;                      // u is the next unit (-1: there is none)
        int3 last1 = make_int3(-1, 0, 0), last2 = last1;       // the two units before
        for (uint32_t it = 0;; ++it) {
            if (!in_hand) {
                u = -1;
                if (phase == 0) {
                    phase = 1;
                    if (ctl->slot < n_units) u = ctl->slot;
                }
                if (u < 0 && phase == 1) {
                    if (n_units > p.b) {
                        if (lane == 0) u = pop_queue(&p.ctrl->die_head[0], p.epoch, n_units - p.b);
                        u = __shfl_sync(0xffffffffu, u, 0);
                        if (u >= 0) u += p.b;
                    }
                    if (u < 0) phase = 2;
                }
                while (u < 0 && scan < p.b) {
                    const int i = scan + lane;
                    const unsigned open = __ballot_sync(0xffffffffu, i < p.b && !slot_taken(p, i));
                    if (!open) {
                        scan += 32;
                        continue;
                    }
                    const int slot = scan + __ffs(open) - 1;
                    int got = 0;
                    if (lane == 0) got = atomicMax(&p.claimed[slot], p.epoch) < p.epoch;
                    got = __shfl_sync(0xffffffffu, got, 0);
                    if (got && slot < n_units) u = slot;
                    scan = slot + 1;
                }
            }
            int3 now = make_int3(-1, 0, 0);        // sequence, KV head, first token
            if (u >= 0) {
                const int e = u / x.H_kv;
                now.y = u - e * x.H_kv;
                int a = 0, b = x.n_seq - 1;
                while (a < b) {
                    const int m = (a + b + 1) >> 1;
                    if (ctl->blocks_before[m] <= e) a = m; else b = m - 1;
                }
                now.x = a;
                now.z = (ctl->blocks_before[a + 1] - 1 - e) * block_tokens;
            }
            // Once everybody has read the unit before this one, the outputs of the one before that are out.
            int ok = 1, second = 0;
            if (lane == 0) {
                if (!mbar_wait_idle(smem_u32(&ctl->unit_empty), (it & 1) ^ 1, abort_flag, limit)) {
                    report_timeout(p, 1);
                    ok = 0;
                }
                second = it >= 2 && *reinterpret_cast<volatile uint32_t*>(&ctl->spoilt[(it - 2) & 3]) == it - 1;
            }
            ok = __shfl_sync(0xffffffffu, ok, 0);
            second = __shfl_sync(0xffffffffu, second, 0);
            if (!ok) break;
            if (second) now = last2;
            in_hand = second || u < 0;
            last2 = last1;
            last1 = now;
            const int seq = now.x, t0 = now.z, head = now.y;
            if (lane == 0) {
                ctl->unit[0] = seq;
                ctl->unit[1] = head;
                ctl->unit[2] = t0;
                ctl->unit[3] = second;
                mbar_arrive(smem_u32(&ctl->unit_full));
            }
            __syncwarp();
            if (seq < 0) {
                if (all_done(it)) break;
                continue;
            }
            const PromptSeq s = ctl->seq[seq];
            for (int w = 0; w < 2; ++w) {
                if (key_tiles(x, s, t0, w) == 0) continue;
                if (lane == 0) {
                    if (!mbar_wait_idle(smem_u32(&ctl->q_empty[w]), (nq[w] & 1) ^ 1, abort_flag, limit)) {
                        report_timeout(p, 2);
                        ok = 0;
                    } else {
                        const uint32_t bar = smem_u32(&ctl->q_full[w]);
                        mbar_expect_tx(bar, x.tpt * x.G * D * 2);
                        for (int d = 0; d < D / 64; ++d)
                            tma_load_3d(q_base + w * C::q_bytes + d * (PA_M * 128), &tm_q, bar, d * 64, head * x.G, s.q0 + t0 + w * x.tpt);
                    }
                }
                ++nq[w];
            }
            ok = __shfl_sync(0xffffffffu, ok, 0);
            if (!ok) break;
        }
    } else if (warp >= 10) {
        // ------------------------------------------------ key tiles (warp 10, even stages) and value tiles (warp 11, odd stages)
        const int which = warp - 10;
        const CUtensorMap* tm = which ? &tm_v : &tm_k;
        uint32_t n = 0, n_tail = 0;                // tiles of this kind so far
        bool ok = true;
        for (uint32_t it = 0; ok; ++it) {
            int seq, head, t0, second;
            if (!next_unit(it, seq, head, t0, second)) break;
            if (seq < 0) {
                if (all_done(it)) break;
                continue;
            }
            const PromptSeq s = ctl->seq[seq];
            const int tiles = max(key_tiles(x, s, t0, 0), key_tiles(x, s, t0, 1));
            const bool scan = which && second;
            if (scan) {                            // (the unit before the one before has been read by everybody: its notes are free)
                for (int i = lane; i < 3 * 128; i += 32) ctl->first_odd[it & 1][0][i] = 0x7fffffff;
                __syncwarp();
            }
            for (int j = 0; j < tiles && ok; ++j, ++n) {
                const uint32_t st = 2 * (n & 1) + which, ph = ((n >> 1) & 1) ^ 1;
                const uint32_t bar = smem_u32(&ctl->kv_full[st]), dst = kv_base + st * C::kv_bytes;
                const int valid = min(s.k_len - j * PA_N, PA_N);
                // The rows behind a sequence's last key belong to the next sequence (or to nothing).  Their scores are masked, but a
                // probability of zero must not meet an infinite or NaN value: the last tile's surplus value rows are cleared.
                const bool clear = which && (valid < PA_N || scan);
                if (!mbar_wait_all(smem_u32(&ctl->kv_empty[st]), ph, abort_flag, limit)) {
                    if (lane == 0) report_timeout(p, 2);
                    ok = false;
                    break;
                }
                const uint32_t land = clear ? smem_u32(&ctl->tail) : bar;
                if (elect_one()) {
                    mbar_expect_tx(land, C::kv_bytes);
#pragma unroll
                    for (int d = 0; d < D / 64; ++d) tma_load_3d(dst + d * (PA_N * 128), tm, land, d * 64, head, s.k0 + j * PA_N);
                }
                __syncwarp();
                if (clear) {
                    if (!mbar_wait_all(land, n_tail & 1, abort_flag, limit)) {
                        if (lane == 0) report_timeout(p, 9);
                        ok = false;
                        break;
                    }
                    ++n_tail;
                    uint8_t* tile = smem + (dst - base);
                    if (scan) take_out_odd<D>(tile, valid, j * PA_N, ctl->first_odd[it & 1]);
#pragma unroll
                    for (int d = 0; d < D / 64; ++d)
                        for (int i = valid * 128 + lane * 16; i < PA_N * 128; i += 512) *reinterpret_cast<uint4*>(tile + d * (PA_N * 128) + i) = make_uint4(0, 0, 0, 0);
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar);
                }
            }
            if (scan && ok && lane == 0) mbar_arrive(smem_u32(&ctl->scanned[it & 1]));
        }
        if (!ok && lane == 0) {
            // gave up: linger (bounded) so that copies already in flight land before the block leaves
            const uint64_t t0 = globaltimer_ns();
            while (globaltimer_ns() - t0 < 2000000ull) __nanosleep(1000);
        }
    } else {
        // ------------------------------------------------ MMA issuer (the warp runs converged, one elected lane issues)
        const uint64_t dk_t = make_smem_desc(0, 16, 1024, 2);                  // Q, K: K-major, 128-byte swizzle
        const uint64_t dv_t = make_smem_desc(0, PA_N * 128, 1024, 2);          // V: N-major, 64-column blocks 16 KB apart
        uint32_t nq[2] = {0, 0}, np[2] = {0, 0}, nk = 0, nv = 0;               // tiles waited for so far
        bool ok = true;
        auto wait = [&](uint64_t* b, uint32_t parity, int role) {
            if (ok && !mbar_wait_all(smem_u32(b), parity, abort_flag, limit)) {
                if (lane == 0) report_timeout(p, role);
                ok = false;
            }
            if (ok) tc_fence_after();
        };
        auto scores = [&](int w, uint32_t st) {
            const uint64_t dq = dk_t | (uint64_t)((q_base + w * C::q_bytes) >> 4), dk = dk_t | (uint64_t)((kv_base + st * C::kv_bytes) >> 4);
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    tc_mma_f16(tmem + w * PA_N, dq + (k >> 2) * (PA_M * 128 >> 4) + (k & 3) * 2, dk + (k >> 2) * (PA_N * 128 >> 4) + (k & 3) * 2, idesc_s, k ? 1u : 0u);
                tc_commit(smem_u32(&ctl->s_full[w]));
            }
            __syncwarp();
        };
        auto commit = [&](uint64_t* b) {
            if (elect_one()) tc_commit(smem_u32(b));
            __syncwarp();
        };
        for (uint32_t it = 0; ok; ++it) {
            int seq, head, t0, second;
            if (!next_unit(it, seq, head, t0, second)) break;
            if (seq < 0) {
                if (all_done(it)) break;
                continue;
            }
            const PromptSeq s = ctl->seq[seq];
            const int n0 = key_tiles(x, s, t0, 0), n1 = key_tiles(x, s, t0, 1), nt = max(n0, n1);
            if (nt == 0) continue;
            uint32_t k_st = 2 * (nk & 1);
            wait(&ctl->kv_full[k_st], (nk >> 1) & 1, 5);
            ++nk;
            for (int w = 0; w < 2 && ok; ++w) {
                const int n = w ? n1 : n0;
                if (n == 0) continue;
                wait(&ctl->q_full[w], nq[w] & 1, 4);
                ++nq[w];
                if (!ok) break;
                scores(w, k_st);
                if (n == 1) commit(&ctl->q_empty[w]);
            }
            if (!ok) break;
            commit(&ctl->kv_empty[k_st]);
            for (int j = 0; j < nt && ok; ++j) {
                const uint32_t v_st = 2 * (nv & 1) + 1;
                wait(&ctl->kv_full[v_st], (nv >> 1) & 1, 5);
                ++nv;
                const bool more = j + 1 < nt;
                if (more) k_st = 2 * (nk & 1);
                bool have_k = false;
                for (int w = 0; w < 2 && ok; ++w) {
                    const int n = w ? n1 : n0;
                    if (j >= n) continue;
                    wait(&ctl->p_full[w], np[w] & 1, 4);
                    ++np[w];
                    if (!ok) break;
                    const uint64_t dv = dv_t | (uint64_t)((kv_base + v_st * C::kv_bytes) >> 4);
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < PA_N / 16; ++k)
                            tc_mma_f16_ts(tmem + 256 + w * D, tmem + w * PA_N + k * 8, dv + k * (2048 >> 4), idesc_o, (j | k) ? 1u : 0u);
                        tc_commit(smem_u32(&ctl->pv_done[w]));
                    }
                    __syncwarp();
                    if (j + 1 < n) {
                        if (!have_k) {
                            wait(&ctl->kv_full[k_st], (nk >> 1) & 1, 5);
                            have_k = true;
                            if (!ok) break;
                        }
                        scores(w, k_st);
                        if (j + 2 == n) commit(&ctl->q_empty[w]);
                    }
                }
                if (!ok) break;
                commit(&ctl->kv_empty[v_st]);
                if (more) {
                    commit(&ctl->kv_empty[k_st]);
                    ++nk;
                }
            }
        }
        __syncwarp();
        if (*abort_flag) {
            // let issued MMAs retire before tensor memory is released
            if (elect_one()) {
                tc_commit(smem_u32(&ctl->mma_drain));
                int dummy = 0;
                mbar_wait(smem_u32(&ctl->mma_drain), 0, &dummy, 2000000ull);
            }
            __syncwarp();
        }
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        // ------------------------------------------------ softmax and epilogue: thread = row of tile w = tensor-memory lane
        const int w = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + lanes + w * PA_N, t_o = tmem + lanes + 256 + w * D;
        const int row_tok = r / x.G, row_head = r - row_tok * x.G;
        const bool wide = (((uintptr_t)x.O | (uintptr_t)(2 * x.o_stride)) & 31) == 0;
        uint32_t ns = 0;                           // score tiles so far = value products so far
        uint32_t scans = 0;                        // parity of the second passes so far, of even units and of odd ones
        bool ok = true;
        for (uint32_t it = 0; ok; ++it) {
            int seq, head, t0, second;
            if (!next_unit(it, seq, head, t0, second)) break;
            if (seq < 0) {
                if (all_done(it)) break;
                continue;
            }
            const PromptSeq s = ctl->seq[seq];
            const int n = key_tiles(x, s, t0, w);
            const int tok = t0 + w * x.tpt + row_tok;
            const bool live = row_tok < x.tpt && tok < s.q_len;
            const int last = last_key(x, s, tok);                              // keys 0 .. last count
            const int all_see = last_key(x, s, t0 + w * x.tpt);                // every row of the tile sees keys 0 .. all_see
            float m = -INFINITY, m_s = 0.f, l = 0.f;                           // reference, times scale (0 for -inf), sum
            for (int j = 0; j < n; ++j, ++ns) {
                if (!mbar_wait_all(smem_u32(&ctl->s_full[w]), ns & 1, abort_flag, limit)) {
                    if (lane == 0) report_timeout(p, 7);
                    ok = false;
                    break;
                }
                tc_fence_after();
                uint32_t sv[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld_32x32(t_s + c * 32, sv[c]);
                tmem_ld_wait();
                if (j * PA_N + PA_N - 1 > all_see) {
                    const int rel = last - j * PA_N;                           // columns 0 .. rel count
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (c * 32 + i > rel) sv[c][i] = 0xff800000u;
                }
                float top4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < 32; ++i)
#pragma unroll
                    for (int c = 0; c < 4; ++c) top4[c] = fmaxf(top4[c], __uint_as_float(sv[c][i]));
                const float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3]));
                const bool grow = top > m && !((top - m) * x.scale_log2e <= PA_LAZY);
                if (j == 0) {
                    m = top;
                } else if (__any_sync(0xffffffffu, grow)) {
                    // the outputs so far are on the old reference: once the last product has landed, move them to the new one
                    if (!mbar_wait_all(smem_u32(&ctl->pv_done[w]), (ns - 1) & 1, abort_flag, limit)) {
                        if (lane == 0) report_timeout(p, 7);
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const float f = !grow ? 1.f : m == -INFINITY ? 0.f : ex2_ftz((m - top) * x.scale_log2e);
                    if (grow) m = top;
                    l *= f;
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        uint32_t ov[32];
                        tmem_ld_32x32(t_o + c, ov);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 32; ++i) ov[i] = __float_as_uint(__uint_as_float(ov[i]) * f);
                        tmem_st_32x32(t_o + c, ov);
                    }
                    tmem_st_wait();
                }
                m_s = m == -INFINITY ? 0.f : m * x.scale_log2e;
                f32x2 sum = pack2(0.f, 0.f);
                const f32x2 scale2 = pack2(x.scale_log2e, x.scale_log2e), ref2 = pack2(-m_s, -m_s);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t pv[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        float a = __uint_as_float(sv[half * 2 + (i >> 4)][(2 * i) & 31]), b = __uint_as_float(sv[half * 2 + (i >> 4)][(2 * i + 1) & 31]);
                        f32x2 v = fma2(pack2(a, b), scale2, ref2);
                        if (i % 8 >= 8 - PA_CUBIC) {
                            v = exp2_cubic(v);
                            unpack2(v, a, b);
                        } else {
                            unpack2(v, a, b);
                            a = ex2_ftz(a);
                            b = ex2_ftz(b);
                            v = pack2(a, b);
                        }
                        sum = add2(sum, v);
                        pv[i] = pack_bf16(a, b);
                    }
                    tmem_st_32x32(t_s + half * 32, pv);
                }
                float sum0, sum1;
                unpack2(sum, sum0, sum1);
                l += sum0 + sum1;
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&ctl->p_full[w]));
            }
            if (!ok) break;
            uint16_t* out = x.O + (size_t)(s.q0 + tok) * x.o_stride + (size_t)(head * x.G + row_head) * D;
            const uint32_t scan_parity = scans >> (it & 1) & 1;
            if (second) scans ^= 1u << (it & 1);
            if (n == 0) {
                if (live)
                    for (int c = 0; c < D; c += 8) *reinterpret_cast<uint4*>(out + c) = make_uint4(0, 0, 0, 0);
                continue;
            }
            if (!mbar_wait_all(smem_u32(&ctl->pv_done[w]), (ns - 1) & 1, abort_flag, limit)) {
                if (lane == 0) report_timeout(p, 7);
                break;
            }
            tc_fence_after();
            const float inv = l == 0.f ? 0.f : 1.f / l;                        // a row that sees no key: zeros
            if (second) {
                // The products are without what is not finite.  What the row sees of that decides: a NaN, or infinities of both signs, make a NaN, one kind
                // of infinity stays, and without any the product stands.  The probabilities are above zero, whatever their rounding.
                if (!mbar_wait_all(smem_u32(&ctl->scanned[it & 1]), scan_parity, abort_flag, limit)) {
                    if (lane == 0) report_timeout(p, 7);
                    break;
                }
                const int(*first_odd)[128] = ctl->first_odd[it & 1];
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t ov[32];
                    tmem_ld_32x32(t_o + c, ov);
                    tmem_ld_wait();
                    if (live) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const bool nan = last >= first_odd[0][c + i], up = last >= first_odd[1][c + i], down = last >= first_odd[2][c + i];
                            float v = __uint_as_float(ov[i]) * inv;
                            if (nan || up || down) v += __uint_as_float(nan || (up && down) ? 0x7fc00000u : up ? 0x7f800000u : 0xff800000u);
                            out[c + i] = (uint16_t)pack_bf16(v, v);
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                continue;
            }
            float odd = 0.f;                                                   // NaN once an output is not finite
#pragma unroll
            for (int c = 0; c < D; c += 32) {
                uint32_t ov[32];
                tmem_ld_32x32(t_o + c, ov);
                tmem_ld_wait();
                if (live) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) odd = fmaf(__uint_as_float(ov[i]), 0.f, odd);
#pragma unroll
                    for (int i = 0; i < 32; i += 16) {
                        uint32_t v[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] = pack_bf16(__uint_as_float(ov[i + 2 * k]) * inv, __uint_as_float(ov[i + 2 * k + 1]) * inv);
                        store32(out + c + i, v, wide);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (__any_sync(0xffffffffu, x.causal && odd != 0.f) && lane == 0) *reinterpret_cast<volatile uint32_t*>(&ctl->spoilt[it & 3]) = it + 1;
        }
    }
    if (!over) {                                   // gave up
        tc_fence_before();
        __syncwarp();
        block_any(true);
    }
    if (warp == 8) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// [tokens][heads][D] with `stride` elements between tokens, box = 64 elements x box_heads x box_tokens, 128-byte swizzle
static bool encode_rows(CUtensorMap* tm, const void* ptr, int D, int heads, long long tokens, long long stride, int box_heads, int box_tokens) {
    EncodeTiledFn enc = get_encode_tiled();
    if (!enc) return false;
    cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)tokens};
    cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)stride * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_tokens};
    cuuint32_t estr[3] = {1, 1, 1};
    return enc(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace ag

using namespace ag;

extern "C" ag_status attention_prompt_persistent(const ag_prompt_attention* a, const ag_plan* plan, void* cuda_stream) {
    if (!a || !plan || a->n_seq < 0 || a->q_tokens < 0 || a->kv_tokens < 0) return AG_ERR_ARG;
    if (a->n_seq == 0 || a->q_tokens == 0) return AG_OK;
    const int G = a->H_kv >= 1 ? a->H_q / a->H_kv : 0;
    const long long most = 1ll << 30;
    if ((a->D != 64 && a->D != 128) || a->H_kv < 1 || a->H_q > 4096 || G < 1 || a->H_q % a->H_kv || G > 64 || a->q_tokens > most || a->kv_tokens > most ||
        !a->Q || !a->O || !a->q_off || (a->kv_tokens > 0 && (!a->K || !a->V)) || !(a->scale >= 0.f) || a->scale > 3.4e38f)
        return AG_ERR_ARG;
    if ((((uintptr_t)a->Q | (uintptr_t)a->K | (uintptr_t)a->V | (uintptr_t)a->O) & 15u) || (((uintptr_t)a->q_off | (uintptr_t)a->kv_off) & 3u)) return AG_ERR_ARG;
    const long long wq = (long long)a->H_q * a->D, wk = (long long)a->H_kv * a->D, far = 1ll << 38;   // a tensor map takes strides below 2^40 bytes
    if (a->q_stride < wq || a->o_stride < wq || a->k_stride < wk || a->v_stride < wk || a->q_stride > far || a->k_stride > far || a->v_stride > far ||
        ((a->q_stride | a->o_stride | a->k_stride | a->v_stride) % 8))
        return AG_ERR_ARG;
    const int tpt = PA_M / G;
    // units are counted in 31 bits
    if ((a->q_tokens / (2 * tpt) + std::min<long long>(a->n_seq, PA_MAXSEQ)) * a->H_kv > 0x7fffffffll) return AG_ERR_ARG;
    ag_status st = check_arch();
    if (st != AG_OK) return st;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    if ((st = refuse_capture(stream)) != AG_OK) return st;
    int dev = 0, n_sm = 0;
    AG_CUDA(cudaGetDevice(&dev));
    AG_CUDA(cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev));
    if (n_sm != plan->lay.n_sm) return AG_ERR_ARG;
    CUtensorMap tm_q, tm_k, tm_v;
    if (!encode_rows(&tm_q, a->Q, a->D, a->H_q, a->q_tokens, a->q_stride, G, tpt)) return AG_ERR_CUDA;
    // without a single key the maps are never used; they are made over Q then
    const bool keys = a->kv_tokens > 0;
    if (!encode_rows(&tm_k, keys ? a->K : a->Q, a->D, keys ? a->H_kv : a->H_q, keys ? a->kv_tokens : a->q_tokens, keys ? a->k_stride : a->q_stride, 1, PA_N) ||
        !encode_rows(&tm_v, keys ? a->V : a->Q, a->D, keys ? a->H_kv : a->H_q, keys ? a->kv_tokens : a->q_tokens, keys ? a->v_stride : a->q_stride, 1, PA_N))
        return AG_ERR_CUDA;
    static std::atomic<unsigned long long> attr_done{0};
    constexpr int smem128 = PCfg<128>::smem_bytes, smem64 = PCfg<64>::smem_bytes > PA_MIN_SMEM ? PCfg<64>::smem_bytes : PA_MIN_SMEM;
    const cudaError_t attr_err = once_per_device(attr_done, [] {
        const cudaError_t e = cudaFuncSetAttribute(k_attn_prompt<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem128);
        return e != cudaSuccess ? e : cudaFuncSetAttribute(k_attn_prompt<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem64);
    });
    if (attr_err != cudaSuccess) return cuda_fail(attr_err);
    PromptArgs x;
    memset(&x, 0, sizeof x);
    x.O = (uint16_t*)a->O;
    x.Q = (const uint16_t*)a->Q; x.K = (const uint16_t*)a->K; x.V = (const uint16_t*)a->V;
    x.q_stride = a->q_stride; x.k_stride = a->k_stride; x.v_stride = a->v_stride; x.o_stride = a->o_stride; x.q_tokens = a->q_tokens; x.kv_tokens = a->kv_tokens;
    x.H_q = a->H_q; x.H_kv = a->H_kv; x.G = G; x.tpt = tpt; x.causal = a->causal ? 1 : 0;
    x.scale_log2e = 1.4426950408889634f * (a->scale > 0.f ? a->scale : 1.f / sqrtf((float)a->D));
    // one launch per PA_MAXSEQ sequences: a block keeps their lengths in shared memory
    for (int s0 = 0; s0 < a->n_seq; s0 += PA_MAXSEQ) {
        x.n_seq = std::min(a->n_seq - s0, PA_MAXSEQ);
        x.q_off = a->q_off + s0;
        x.kv_off = (a->kv_off ? a->kv_off : a->q_off) + s0;
        if ((st = renew_epochs_if_needed(plan, stream)) != AG_OK) return st;
        PersistParams gp = make_persist_params(plan, 0, 0, 0);
        gp.wait_limit_ns += 200ull * a->kv_tokens;       // a wait may last a unit: up to 17 us for 128 keys (second pass, D = 128)
        const unsigned grid = plan->grid_blocks > 0 ? plan->grid_blocks : plan->lay.n_sm;
        if (a->D == 128) k_attn_prompt<128><<<grid, PA_THREADS, smem128, stream>>>(tm_q, tm_k, tm_v, gp, x);
        else k_attn_prompt<64><<<grid, PA_THREADS, smem64, stream>>>(tm_q, tm_k, tm_v, gp, x);
        const cudaError_t le = cudaGetLastError();
        if (le != cudaSuccess) return launch_failed(plan, le);
        count_launch();
    }
    return AG_OK;
}
