// Rotary positions: heads turned by the angles of their token's position, and a step's new keys and values on their way into the 4-bit cache.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "kv4.cuh"

namespace ag {

// A warp has one token (or a stretch of its heads): D / 16 lanes hold a row, sixteen elements each, so that a warp takes 4 (D = 128) or 8 rows at a time, and every lane
// keeps the cosines and sines of its eight pairs in registers for all heads of the token.  The angles' 64-bit cosines and sines are shared out over the lanes.
//   a' = a c - b s,  b' = b c + a s      a c and b c rounded to 32 bits, the rest by one multiply-add, two at a time
// "Halves": a lane has the two chunks of eight elements that are turned with one another, rot / 2 apart (the lanes behind those have neighbouring chunks, which stay);
// "pairs": two neighbouring chunks.  Quantisation wants neighbouring chunks, so keys on their way into the cache are passed from lane to lane once they have been turned.
// Bound: memory, and the latency of its loads where the angles wait in front of them: three blocks on an SM (80 registers) turn 16384 tokens x 40 heads in 55 us (6.1 TB/s, 0.93 of a
// copy), two (94 registers) in 58, four spill and take 63; appended and loaded back 87, 95 and 95.  A step of Q is 60 instructions; with the chunks of a lane side by side, partners fetched
// from other lanes and one element at a time it was 320, and the same tokens took 76 us.
constexpr int RO_THREADS = 256;
constexpr int RO_WARPS = RO_THREADS / 32;
constexpr int RO_ROWS = 4;                 // steps whose loads are in flight together

struct RotaryArgs {
    const uint16_t *Q, *K, *V;
    uint16_t *Q_out, *K_out;
    long long q_stride, k_stride, v_stride, q_out_stride, k_out_stride, n_tokens, n_rows;
    const int32_t *pos, *from, *slot;
    const double* freq;
    double magnitude;
    uint8_t* pages;
    long long n_slots;
    int H_q, H_kv, rot, pairs;
    int q_steps, k_steps, v_steps, parts;  // steps of 512 / D heads; stretches that a token's steps are cut into
};

// the lane's pairs (w[0 .. 3] with w[4 .. 7], or the halves of a word) turned
template <bool PAIRS>
__device__ __forceinline__ void turn(uint32_t (&w)[8], const f32x2 (&c)[4], const f32x2 (&s)[4], const f32x2 (&minus_s)[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        // four elements of pairs 2 k and 2 k + 1 of the lane: a in x, b in y
        uint32_t u = w[PAIRS ? 2 * k : k], v = w[PAIRS ? 2 * k + 1 : 4 + k];
        const f32x2 x = PAIRS ? pack2(bf16_lo(u), bf16_lo(v)) : pack2(bf16_lo(u), bf16_hi(u)), y = PAIRS ? pack2(bf16_hi(u), bf16_hi(v)) : pack2(bf16_lo(v), bf16_hi(v));
        float a0, a1, b0, b1;
        unpack2(fma2(y, minus_s[k], mul2(x, c[k])), a0, a1);
        unpack2(fma2(x, s[k], mul2(y, c[k])), b0, b1);
        w[PAIRS ? 2 * k : k] = PAIRS ? pack_bf16(a0, b0) : pack_bf16(a0, a1);
        w[PAIRS ? 2 * k + 1 : 4 + k] = PAIRS ? pack_bf16(a1, b1) : pack_bf16(b0, b1);
    }
}

template <int D, bool PAIRS>
__global__ void __launch_bounds__(RO_THREADS, 3) k_rotary(const RotaryArgs x) {
    constexpr int L = D / 16, ROWS = 32 / L, U = RO_ROWS;
    __shared__ float2 turns[RO_WARPS][D / 2];
    dep_wait();
    dep_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane % L;
    const long long item = (long long)blockIdx.x * RO_WARPS + warp, token = item / x.parts;
    if (token >= x.n_tokens) return;
    const int part = (int)(item - token * x.parts), steps = x.q_steps + x.k_steps + x.v_steps;
    const int first = (int)((long long)steps * part / x.parts), end = (int)((long long)steps * (part + 1) / x.parts);
    const long long row = x.from ? x.from[token] : token;
    if (x.from && (row < 0 || row >= x.n_rows)) return;
    const int at = x.slot ? x.slot[token] : -1;
    uint8_t* page = at >= 0 && at < x.n_slots ? x.pages + (size_t)(at / KV4_PAGE) * x.H_kv * kv4_head_bytes(D) : nullptr;

    // the lane's chunks
    const int o = x.rot / 16;
    const bool turned = l < o;                                 // (pairs: chunks 2 l and 2 l + 1 of the first 2 o; halves: l and l + o)
    const int e0 = !PAIRS && turned ? 8 * l : 16 * l, e1 = !PAIRS && turned ? 8 * (l + o) : 16 * l + 8;
    auto load = [&](const uint16_t* rows, int f0, int f1, int head, int heads, int st, int st_end, uint32_t(&w)[8]) {
        uint4 a = make_uint4(0, 0, 0, 0), b = a;
        if (head < heads && st < st_end) {
            a = *reinterpret_cast<const uint4*>(rows + head * D + f0);
            b = *reinterpret_cast<const uint4*>(rows + head * D + f1);
        }
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
        w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    };
    auto store = [&](uint16_t* rows, int head, const uint32_t(&w)[8]) {
        *reinterpret_cast<uint4*>(rows + head * D + e0) = make_uint4(w[0], w[1], w[2], w[3]);
        *reinterpret_cast<uint4*>(rows + head * D + e1) = make_uint4(w[4], w[5], w[6], w[7]);
    };
    const int q0 = min(first, x.q_steps), q1 = min(end, x.q_steps), k0 = max(first - x.q_steps, 0), k1 = min(end - x.q_steps, x.k_steps);
    const int v0 = max(first - x.q_steps - x.k_steps, 0), v1 = end - x.q_steps - x.k_steps;
    const uint16_t *q_rows = x.Q + row * x.q_stride, *k_rows = x.K + row * x.k_stride, *v_rows = x.V + row * x.v_stride;
    uint32_t w[U][8];
    if (q0 < q1) {                                             // (on their way while the angles are taken)
#pragma unroll
        for (int u = 0; u < U; ++u) load(q_rows, e0, e1, (q0 + u) * ROWS + lane / L, x.H_q, q0 + u, q1, w[u]);
    }
    f32x2 c[4], s[4], minus_s[4];
    if (x.rot && first < x.q_steps + x.k_steps) {
        const double pos = (double)x.pos[token];
        for (int i = lane; i < x.rot / 2; i += 32) {
            double sn, cs;
            sincos(pos * x.freq[i], &sn, &cs);
            turns[warp][i] = make_float2((float)(cs * x.magnitude), (float)(sn * x.magnitude));
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 t0 = turns[warp][turned ? 8 * l + 2 * k : 0], t1 = turns[warp][turned ? 8 * l + 2 * k + 1 : 0];
            c[k] = pack2(t0.x, t1.x);
            s[k] = pack2(t0.y, t1.y);
            minus_s[k] = pack2(-t0.y, -t1.y);
        }
    }
    for (int st = q0; st < q1; st += U) {
        if (st > q0) {
#pragma unroll
            for (int u = 0; u < U; ++u) load(q_rows, e0, e1, (st + u) * ROWS + lane / L, x.H_q, st + u, q1, w[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int head = (st + u) * ROWS + lane / L;
            if (turned) turn<PAIRS>(w[u], c, s, minus_s);
            if (st + u < q1 && head < x.H_q) store(x.Q_out + token * x.q_out_stride, head, w[u]);
        }
    }
    for (int st = k0; st < k1; st += 2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) load(k_rows, e0, e1, (st + u) * ROWS + lane / L, x.H_kv, st + u, k1, w[u]);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int head = (st + u) * ROWS + lane / L;
            const bool live = st + u < k1 && head < x.H_kv;
            if (turned) turn<PAIRS>(w[u], c, s, minus_s);
            if (x.K_out && live) store(x.K_out + token * x.k_out_stride, head, w[u]);
            if (!x.pages) continue;
            uint32_t in[8];
            if (PAIRS || !x.rot) {
#pragma unroll
                for (int k = 0; k < 8; ++k) in[k] = w[u][k];
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {                  // chunk 2 l + h is with another lane, as its first chunk or its second
                    const int chunk = 2 * l + h, from = lane - l + (chunk < o ? chunk : chunk < 2 * o ? chunk - o : chunk >> 1);
                    const bool second = chunk < 2 * o ? chunk >= o : chunk & 1;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t a = __shfl_sync(0xffffffffu, w[u][k], from), b = __shfl_sync(0xffffffffu, w[u][4 + k], from);
                        in[4 * h + k] = second ? b : a;
                    }
                }
            }
            uint32_t codes[2];
            const uint32_t pair = kv4_quantise<D>(in, 0, l, codes);
            if (live && page) kv4_put<D>(page + (size_t)head * kv4_head_bytes(D), 0, at % KV4_PAGE, l, codes, pair);
        }
    }
    for (int st = v0; st < v1; st += 2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) load(v_rows, 16 * l, 16 * l + 8, (st + u) * ROWS + lane / L, x.H_kv, st + u, v1, w[u]);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int head = (st + u) * ROWS + lane / L;
            uint32_t codes[2];
            const uint32_t pair = kv4_quantise<D>(w[u], 1, l, codes);
            if (st + u < v1 && head < x.H_kv && page) kv4_put<D>(page + (size_t)head * kv4_head_bytes(D), 1, at % KV4_PAGE, l, codes, pair);
        }
    }
}

static bool row_ok(const void* p, int64_t stride, int H, int D) {
    return p && !((uintptr_t)p & 15u) && H >= 1 && H <= 4096 && stride >= (int64_t)H * D && stride % 8 == 0;
}

static ag_status rotary_rows(const ag_kv4_pool* pool, const ag_rotary* r, const ag_rotary_rows* x, const int32_t* slot, void* cuda_stream) {
    if (!x || x->n_tokens < 0 || x->n_tokens > (1ll << 31) - 1) return AG_ERR_ARG;
    const int D = pool ? pool->D : x->D, H_kv = pool ? pool->H_kv : x->H_kv;
    if (D != 64 && D != 128) return AG_ERR_ARG;
    if (r && (!r->freq || ((uintptr_t)r->freq & 7u) || r->rot < 16 || r->rot > D || r->rot % 16 || (r->layout != AG_ROTARY_HALVES && r->layout != AG_ROTARY_PAIRS) ||
              !(fabs(r->magnitude) <= 1e30)))
        return AG_ERR_ARG;
    if (x->n_tokens == 0) return AG_OK;
    const bool q = x->Q || x->Q_out, k = x->K || x->K_out;
    if (!q && !k) return AG_ERR_ARG;
    if (q && (!row_ok(x->Q, x->q_stride, x->H_q, D) || !row_ok(x->Q_out, x->q_out_stride, x->H_q, D))) return AG_ERR_ARG;
    if (k && (!row_ok(x->K, x->k_stride, H_kv, D) || ((x->K_out || !pool) && !row_ok(x->K_out, x->k_out_stride, H_kv, D)))) return AG_ERR_ARG;
    if (pool && (!k || !row_ok(x->V, x->v_stride, H_kv, D) || !slot || ((uintptr_t)slot & 3u))) return AG_ERR_ARG;
    if ((r && !x->pos) || (((uintptr_t)x->pos | (uintptr_t)x->from) & 3u) || (x->from && x->n_rows < 0)) return AG_ERR_ARG;
    // in place: the same rows only
    if (q && x->Q_out == x->Q && (x->from || x->q_out_stride != x->q_stride)) return AG_ERR_ARG;
    if (x->K_out && x->K_out == x->K && (x->from || x->k_out_stride != x->k_stride)) return AG_ERR_ARG;
    if (x->K_out && (x->K_out == x->Q_out || x->K_out == x->Q || x->K_out == x->V)) return AG_ERR_ARG;
    if (q && (x->Q_out == x->K || (pool && x->Q_out == x->V))) return AG_ERR_ARG;
    ag_status st = check_arch();
    if (st != AG_OK) return st;
    RotaryArgs a;
    memset(&a, 0, sizeof a);
    a.Q = (const uint16_t*)x->Q; a.K = (const uint16_t*)x->K; a.V = (const uint16_t*)x->V;
    a.Q_out = (uint16_t*)x->Q_out; a.K_out = (uint16_t*)x->K_out;
    a.q_stride = x->q_stride; a.k_stride = x->k_stride; a.v_stride = x->v_stride; a.q_out_stride = x->q_out_stride; a.k_out_stride = x->k_out_stride;
    a.n_tokens = x->n_tokens; a.n_rows = x->n_rows;
    a.pos = x->pos; a.from = x->from; a.slot = pool ? slot : nullptr;
    if (r) {
        a.freq = r->freq; a.magnitude = r->magnitude; a.rot = r->rot; a.pairs = r->layout == AG_ROTARY_PAIRS;
    }
    if (pool) {
        a.pages = (uint8_t*)pool->pages;
        a.n_slots = (long long)pool->n_pages * KV4_PAGE;
    }
    a.H_q = q ? x->H_q : 0; a.H_kv = k ? H_kv : 0;
    const int rows = 512 / D;
    a.q_steps = (a.H_q + rows - 1) / rows;
    a.k_steps = (a.H_kv + rows - 1) / rows;
    a.v_steps = pool ? a.k_steps : 0;
    const int steps = a.q_steps + a.k_steps + a.v_steps;
    // few tokens are cut by heads, down to one step a warp, until every SM has its sixteen warps
    a.parts = (int)std::max<long long>(1, std::min<long long>(steps, 148ll * 16 / x->n_tokens));
    const long long blocks = (x->n_tokens * a.parts + RO_WARPS - 1) / RO_WARPS;
    if (blocks > 0x7fffffffll) return AG_ERR_ARG;
    void (*kernel)(RotaryArgs) = D == 128 ? (a.pairs ? k_rotary<128, true> : k_rotary<128, false>) : (a.pairs ? k_rotary<64, true> : k_rotary<64, false>);
    AG_CUDA(launch_dependent(kernel, (unsigned)blocks, RO_THREADS, reinterpret_cast<cudaStream_t>(cuda_stream), a));
    count_launch();
    return AG_OK;
}

}  // namespace ag

using namespace ag;

extern "C" ag_status ag_rotary_apply(const ag_rotary* r, const ag_rotary_rows* x, void* cuda_stream) {
    if (!r) return AG_ERR_ARG;
    return rotary_rows(nullptr, r, x, nullptr, cuda_stream);
}

extern "C" ag_status ag_kv4_append_rotary(const ag_kv4_pool* pool, const ag_rotary* r, const ag_rotary_rows* x, const int32_t* slot, void* cuda_stream) {
    if (!kv4_pool_ok(pool)) return AG_ERR_ARG;
    return rotary_rows(pool, r, x, slot, cuda_stream);
}

extern "C" ag_status ag_rotary_frequencies(const ag_rotary_scaling* s, double* freq, double* magnitude) {
    if (!s || !freq || !magnitude || s->rot < 2 || s->rot > 1024 || s->rot % 2 || !(s->base > 1.0 && s->base < 1e300) || s->scaling < AG_ROTARY_PLAIN ||
        s->scaling > AG_ROTARY_RAMP)
        return AG_ERR_ARG;
    if (s->scaling != AG_ROTARY_PLAIN && !(s->factor >= 1.0 && s->factor < 1e30)) return AG_ERR_ARG;
    const bool by_turns = s->scaling == AG_ROTARY_BANDS || s->scaling == AG_ROTARY_RAMP;
    if (by_turns && !(s->context > 0.0 && s->context < 1e30 && s->low > 0.0 && s->low < s->high && s->high < 1e30)) return AG_ERR_ARG;
    const double two_pi = 6.283185307179586476925286766559;
    double a = 0, b = 0;
    *magnitude = 1.0;
    if (s->scaling == AG_ROTARY_RAMP) {
        auto place = [&](double turns) { return s->rot * log(s->context / (two_pi * turns)) / (2.0 * log(s->base)); };
        a = std::max(0.0, floor(place(s->high)));
        b = std::min((double)(s->rot - 1), ceil(place(s->low)));
        *magnitude = 0.1 * log(s->factor) + 1.0;
    }
    for (int i = 0; i < s->rot / 2; ++i) {
        const double f = pow(s->base, -2.0 * i / s->rot);
        double keep = 1.0;                                    // share of the frequency that stays
        if (s->scaling == AG_ROTARY_LINEAR) keep = 0.0;
        else if (s->scaling == AG_ROTARY_BANDS) keep = (s->context * f / two_pi - s->low) / (s->high - s->low);
        else if (s->scaling == AG_ROTARY_RAMP) keep = 1.0 - (i - a) / std::max(b - a, 0.001);
        keep = std::min(1.0, std::max(0.0, keep));
        freq[i] = s->scaling == AG_ROTARY_PLAIN ? f : f * keep + f / s->factor * (1.0 - keep);
    }
    return AG_OK;
}
