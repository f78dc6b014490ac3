// Rotary positions: heads turned by the angles of their token's position, and a step's new keys and values on their way into the 4-bit cache.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "kv4.cuh"

namespace ag {

// A warp has one token (or a stretch of its heads): D / 16 lanes hold a row, sixteen elements each, as in the store of the cache, so that a warp takes 4 (D = 128)
// or 8 rows at a time, and every lane keeps the cosines and sines of its sixteen elements in registers for all heads of the token.  The angles' 64-bit
// cosines and sines are shared out over the lanes, two each at rot = 128: one in six of the warp's issue slots for 48 heads.
//   a' = a c - b s,  b' = b c + a s
// both as own * c + partner * s' (s' = -s for the first of a pair), every product and the sum rounded to 32 bits.  The partner of an element is in the same word
// ("pairs") or comes from another lane ("halves"), where it lies rot / 16 eight-element chunks away.
constexpr int RO_THREADS = 256;
constexpr int RO_WARPS = RO_THREADS / 32;
constexpr int RO_ROWS = 2;                 // steps whose loads are in flight together

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

template <int D, bool PAIRS>
__global__ void __launch_bounds__(RO_THREADS) k_rotary(const RotaryArgs x) {
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

    uint4 raw[U][2];
    // step st: its kind (0 Q, 1 K, 2 V) and the lane's head
    auto kind_of = [&](int st) { return st < x.q_steps ? 0 : st < x.q_steps + x.k_steps ? 1 : 2; };
    auto head_of = [&](int st, int kind) { return (st - (kind == 0 ? 0 : kind == 1 ? x.q_steps : x.q_steps + x.k_steps)) * ROWS + lane / L; };
    auto load = [&](int st, uint4 (&to)[2]) {
        to[0] = to[1] = make_uint4(0, 0, 0, 0);
        if (st >= end) return;
        const int kind = kind_of(st), head = head_of(st, kind);
        if (head >= (kind == 0 ? x.H_q : x.H_kv)) return;
        const uint16_t* p = (kind == 0 ? x.Q + row * x.q_stride : kind == 1 ? x.K + row * x.k_stride : x.V + row * x.v_stride) + head * D + l * 16;
        to[0] = reinterpret_cast<const uint4*>(p)[0];
        to[1] = reinterpret_cast<const uint4*>(p)[1];
    };
#pragma unroll
    for (int u = 0; u < U; ++u) load(first + u, raw[u]);

    // the token's cosines and sines, then the lane's own
    const int half = x.rot / 2, o = x.rot / 16;
    constexpr int N = PAIRS ? 8 : 16;
    float c[N], s[N];
    if (x.rot && first < x.q_steps + x.k_steps) {
        const double pos = (double)x.pos[token];
        for (int i = lane; i < half; i += 32) {
            double sn, cs;
            sincos(pos * x.freq[i], &sn, &cs);
            turns[warp][i] = make_float2((float)(cs * x.magnitude), (float)(sn * x.magnitude));
        }
        __syncwarp();
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int e = l * 16 + (PAIRS ? 2 * j : j);
            const float2 t = turns[warp][e >= x.rot ? 0 : PAIRS ? e >> 1 : e < half ? e : e - half];
            c[j] = t.x;
            s[j] = !PAIRS && e < half ? -t.y : t.y;
        }
    }
    for (int st0 = first; st0 < end; st0 += U) {
        uint32_t in[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t v[8] = {raw[u][0].x, raw[u][0].y, raw[u][0].z, raw[u][0].w, raw[u][1].x, raw[u][1].y, raw[u][1].z, raw[u][1].w};
#pragma unroll
            for (int k = 0; k < 8; ++k) in[u][k] = v[k];
            load(st0 + U + u, raw[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int st = st0 + u;
            if (st >= end) break;
            const int kind = kind_of(st), head = head_of(st, kind);
            const bool live = head < (kind == 0 ? x.H_q : x.H_kv);
            if (kind < 2 && x.rot) {
                if (PAIRS) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float a = bf16_lo(in[u][j]), b = bf16_hi(in[u][j]);
                        const uint32_t w = pack_bf16(__fsub_rn(__fmul_rn(a, c[j]), __fmul_rn(b, s[j])), __fadd_rn(__fmul_rn(b, c[j]), __fmul_rn(a, s[j])));
                        if (l * 16 + 2 * j < x.rot) in[u][j] = w;
                    }
                } else {
                    const bool odd = o & 1;
                    uint32_t other[8];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {                  // chunk 2 l + h; its partner o chunks up or down
                        const int chunk = 2 * l + h, partner = chunk < o ? chunk + o : chunk < 2 * o ? chunk - o : chunk;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            other[4 * h + k] = __shfl_sync(0xffffffffu, odd ? in[u][4 * (1 - h) + k] : in[u][4 * h + k], lane - l + (partner >> 1));
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float a = __fadd_rn(__fmul_rn(bf16_lo(in[u][k]), c[2 * k]), __fmul_rn(bf16_lo(other[k]), s[2 * k]));
                        const float b = __fadd_rn(__fmul_rn(bf16_hi(in[u][k]), c[2 * k + 1]), __fmul_rn(bf16_hi(other[k]), s[2 * k + 1]));
                        if (l * 16 + 2 * k < x.rot) in[u][k] = pack_bf16(a, b);
                    }
                }
            }
            uint16_t* out = kind == 0 ? x.Q_out : kind == 1 ? x.K_out : nullptr;
            if (out && live) {
                out += token * (kind == 0 ? x.q_out_stride : x.k_out_stride) + head * D + l * 16;
                reinterpret_cast<uint4*>(out)[0] = make_uint4(in[u][0], in[u][1], in[u][2], in[u][3]);
                reinterpret_cast<uint4*>(out)[1] = make_uint4(in[u][4], in[u][5], in[u][6], in[u][7]);
            }
            if (kind > 0 && x.pages) {
                uint32_t w[2];
                const uint32_t pair = kv4_quantise<D>(in[u], kind - 1, l, w);
                if (live && at >= 0 && at < x.n_slots)
                    kv4_put<D>(x.pages + ((size_t)(at / KV4_PAGE) * x.H_kv + head) * kv4_head_bytes(D), kind - 1, at % KV4_PAGE, l, w, pair);
            }
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
