// Log probabilities of given tokens, their gradient with respect to the logits, and the most probable tokens of a row: what a model
// gives to tokens that are there already, where the sampling kernels draw new ones.
//
// With l = logits / T, p = softmax(l) over all tokens, q = softmax(l) over the valid ones (q = p without a mask), t the row's token:
//   log q_t        = l_t - log sum_valid e^l
//   log Z_valid    = log sum_valid e^l - log sum e^l
//   entropy        = -sum q log q = log S - (sum y e^y) / S       with y = l - reference, S = sum e^y over the valid tokens
//   d_l            = d_logprob (1[v = t] - q) + d_logZ (q - p) - d_entropy q (log q + entropy),   d_logits = d_l / T
// A row is read once, by all lanes of its wavefronts, each with its own running reference (the largest logit it has seen) and sums
// relative to it; the lanes' sums are brought to one reference at the end.  Differences of logits are taken before they are
// multiplied, so that rows far from 0 lose nothing.  Sums are fp32: a lane adds at most 4,096 terms of one sign.
#include "ppv_rows.h"

namespace {

constexpr int MOST_WAVES = 16;       // wavefronts per row and workgroup
constexpr int SHORT_ROWS = 4;        // rows of one tile: so many to a workgroup, a wavefront each
constexpr unsigned MOST_GROUPS = 1u << 20;   // workgroups of a launch: more rows than that are taken in turns
constexpr float LOWEST = -3.402823466e38f;
constexpr float FAINT = -1000.f;     // as an exponent of 2: a weight of 0

// ------------------------------------------------------------------------------------------
// Sums over tokens: reference m, s = sum 2^((x - m) c), w = sum of each of these times its exponent.  An empty sum has m = LOWEST, which
// is finite: no difference below is that of two infinities.
struct Sums {
    float m, s, w;
};
__device__ __forceinline__ Sums no_sums() { return {LOWEST, 0.f, 0.f}; }
__device__ __forceinline__ float most(float a, float b) {   // (without the instruction that quiets a NaN first)
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ float most(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
// sums relative to the reference m, which is not below their own
template <bool W> __device__ __forceinline__ void refer(Sums &a, float m, float c) {
    const float d = most((a.m - m) * c, FAINT), f = fast_exp2(d);
    if (W) a.w = f * fmaf(d, a.s, a.w);
    a.s *= f;
    a.m = m;
}
template <int N, bool W> __device__ __forceinline__ void take(Sums &a, const float (&x)[N], float c) {
    float m = a.m;
#pragma unroll
    for (int i = 0; i < N; i += 2) m = most(m, x[i], x[i + 1]);
    refer<W>(a, m, c);
#pragma unroll
    for (int i = 0; i < N; i++) {
        const float y = (x[i] - m) * c, e = fast_exp2(y);
        a.s += e;
        if (W) a.w = fmaf(most(y, FAINT), e, a.w);   // (-inf: nothing, not a NaN)
    }
}
template <bool W> __device__ __forceinline__ Sums over_wave(Sums a, float c) {
    refer<W>(a, wave_max(a.m), c);
    a.s = wave_sum(a.s);
    if (W) a.w = wave_sum(a.w);
    return a;
}

// A row's mask as the memory unit's buffer; what is asked for behind its end is 0.
__device__ __forceinline__ Row mask_of(const uint32_t *mask, int64_t b, int n_words) {
    return row_of<uint32_t, 0u>(mask + b * n_words, n_words);
}
// Bits of this lane's tokens of load j of a tile: their byte (bf16), or half of it.
template <typename T> __device__ __forceinline__ uint32_t bits_raw(const Row &mask, int tile, int j, int lane) {
    const uint32_t v = (uint32_t)tile * TileGeom<T>::TILE + (uint32_t)j * TileGeom<T>::PER_LOAD + (uint32_t)lane * TileGeom<T>::EPL;
    return __builtin_amdgcn_raw_buffer_load_b8(mask.buf, v >> 3, 0, 0);
}
template <typename T> __device__ __forceinline__ uint32_t bits_fix(uint32_t raw, int lane) {
    return TileGeom<T>::EPL == 8 ? raw : (raw >> ((lane & 1) * 4)) & 0xFu;
}
__device__ __forceinline__ float if_bit(float x, uint32_t bits, int k) { return (bits >> k) & 1u ? x : -INFINITY; }

template <typename T> struct MaskedTile {
    RawTile t;
    uint32_t bits[4];
    template <bool MASK> __device__ __forceinline__ void load(const Row &row, const Row &mask, int tile, int lane) {
        load_tile<T>(row, tile, lane, t);
        if (MASK) {
#pragma unroll
            for (int j = 0; j < 4; j++) bits[j] = bits_raw<T>(mask, tile, j, lane);
        }
    }
};
template <typename T, bool PAD> __device__ __forceinline__ void unpack_group(const u32x4 &r, int left, float (&x)[Elem<T>::EPL]) {
    Elem<T>::unpack(r, x);
    if (PAD) {
#pragma unroll
        for (int k = 0; k < Elem<T>::EPL; k++) x[k] = k < left ? x[k] : -INFINITY;
    }
}

// One tile's tokens into the sums over all tokens and, with a mask, over the valid ones.  ALL: the former are wanted.
template <typename T, bool MASK, bool ALL, bool W, bool PAD>
__device__ __forceinline__ void take_tile(const MaskedTile<T> &mt, int left, int lane, float c, Sums &all, Sums &valid) {
    constexpr int EPL = Elem<T>::EPL;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        float x[EPL];
        unpack_group<T, PAD>(mt.t.r[j], left - j * TileGeom<T>::PER_LOAD, x);
        if (ALL) take<EPL, W && !MASK>(all, x, c);
        if (MASK) {
            const uint32_t bits = bits_fix<T>(mt.bits[j], lane);
            if (__ballot(bits != 0u) != 0ull) {
#pragma unroll
                for (int k = 0; k < EPL; k++) x[k] = if_bit(x[k], bits, k);
                take<EPL, W>(valid, x, c);
            }
        }
    }
}
// The tiles first, first + step, ... of a row
template <typename T, bool MASK, bool ALL, bool W>
__device__ __forceinline__ void take_row(const Row &row, const Row &mask, int V, int first, int step, int lane, float c, Sums &all, Sums &valid) {
    const int nt = (V + TileGeom<T>::TILE - 1) / TileGeom<T>::TILE;
    MaskedTile<T> now, next;
    now.template load<MASK>(row, mask, first, lane);
    for (int t = first; t < nt; t += step) {
        next.template load<MASK>(row, mask, t + step, lane);   // (behind the row: nothing is read)
        const int left = tokens_left<T>(V, t, lane);
        if ((t + 1) * TileGeom<T>::TILE <= V) take_tile<T, MASK, ALL, W, false>(now, left, lane, c, all, valid);
        else take_tile<T, MASK, ALL, W, true>(now, left, lane, c, all, valid);
        now = next;
    }
}

// Sums of a workgroup's wavefronts, to every wavefront.
struct RowSums {
    Sums all[MOST_WAVES], valid[MOST_WAVES];
    float x;   // the row's token's logit
};
template <bool W> __device__ __forceinline__ Sums over_waves(const Sums *part, int nw, int lane, float c) {
    return over_wave<W>(lane < nw ? part[lane] : no_sums(), c);
}

// The row's token's logit; -inf where there is no such token, or it is not valid.
template <typename T> __device__ __forceinline__ float logit_of(const T *row, const uint32_t *mask_row, int tok, int V) {
    if ((uint32_t)tok >= (uint32_t)V) return -INFINITY;
    if (mask_row && !((mask_row[tok >> 5] >> (tok & 31)) & 1u)) return -INFINITY;
    return sizeof(T) == 4 ? ((const float *)row)[tok] : __uint_as_float((uint32_t)((const uint16_t *)row)[tok] << 16);
}

struct Outputs {
    float *logprobs, *logZ_valid, *entropy, *stats;
};
struct RowValues {
    float logprob, logZ, entropy;
};
// what the sums say.  Without mass (no valid token, or all at -inf): -inf, and an entropy of 0.
template <bool MASK> __device__ __forceinline__ RowValues row_values(const Sums &all, const Sums &q, float x, const Temper &tp) {
    if (!(q.s != 0.f)) return {-INFINITY, -INFINITY, 0.f};
    const float log_s = logf(q.s);
    return {(x - q.m) * tp.inv - log_s, MASK ? fmaf(q.m - all.m, tp.inv, log_s - logf(all.s)) : 0.f,
            fmaxf(fmaf(q.w / q.s, -LN2F, log_s), 0.f)};
}
__device__ __forceinline__ void put_stats(float *stats, int64_t b, const Sums &all, const Sums &q, const RowValues &v) {
    float4 *at = (float4 *)(stats + b * PPV_LOGPROB_STATS);
    at[0] = {all.m, all.s, q.m, q.s};
    at[1] = {v.entropy, v.logprob, 0.f, 0.f};
}
__device__ __forceinline__ void put_values(const Outputs &o, int64_t b, const RowValues &v) {
    if (o.logprobs) o.logprobs[b] = v.logprob;
    if (o.logZ_valid) o.logZ_valid[b] = v.logZ;
    if (o.entropy) o.entropy[b] = v.entropy;
}

// ------------------------------------------------------------------------------------------
// Forward.  ONE: rows of one tile, a wavefront each; else a workgroup has a row.
template <typename T, bool MASK, bool W, bool ONE>
__global__ __launch_bounds__(ONE ? SHORT_ROWS *WAVE : MOST_WAVES *WAVE) void score_kernel(const T *__restrict__ logits, int64_t row_stride,
                                                                                         const int32_t *__restrict__ tokens, const uint32_t *__restrict__ mask,
                                                                                         int V, int n_words, int B, Outputs out, Temper tp) {
    __shared__ RowSums sh;
    const int lane = threadIdx.x & (WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), nw = ONE ? 1 : blockDim.x / WAVE;
    const int per = ONE ? SHORT_ROWS : 1;
    for (int64_t b = (int64_t)blockIdx.x * per + (ONE ? wave : 0); b < B; b += (int64_t)gridDim.x * per) {
        const int tok = tokens ? tokens[b] : 0;
        if (tok < 0) {   // left out
            if (ONE ? lane == 0 : threadIdx.x == 0) {
                put_values(out, b, {0.f, 0.f, 0.f});
                if (out.stats) put_stats(out.stats, b, {0.f, 0.f, 0.f}, {0.f, 0.f, 0.f}, {0.f, 0.f, 0.f});
            }
            continue;
        }
        const T *at = logits + b * row_stride;
        const Row row = row_of(at, V), mrow = MASK ? mask_of(mask, b, n_words) : row;
        const float x = tokens ? logit_of(at, MASK ? mask + b * n_words : nullptr, tok, V) : -INFINITY;
        Sums all = no_sums(), valid = no_sums();
        take_row<T, MASK, true, W>(row, mrow, V, ONE ? 0 : wave, nw, lane, tp.c, all, valid);
        all = over_wave<W && !MASK>(all, tp.c);
        if (MASK) valid = over_wave<W>(valid, tp.c);
        if (!ONE) {
            if (lane == 0) {
                sh.all[wave] = all;
                if (MASK) sh.valid[wave] = valid;
            }
            __syncthreads();
            if (wave == 0) {
                all = over_waves<W && !MASK>(sh.all, nw, lane, tp.c);
                if (MASK) valid = over_waves<W>(sh.valid, nw, lane, tp.c);
            }
        }
        if (lane == 0 && (ONE || wave == 0)) {
            const Sums q = MASK ? valid : all;
            const RowValues v = row_values<MASK>(all, q, x, tp);
            put_values(out, b, v);
            if (out.stats) put_stats(out.stats, b, all, q, v);
        }
        if (!ONE) __syncthreads();   // before LDS is used again
    }
}

// ------------------------------------------------------------------------------------------
// Gradient.
struct Upstream {
    const float *logprobs, *logZ_valid, *entropy;
};
// d_logits = e_q (a + b y_q) - z e_p, and `at_token` more at the row's token; e_q = 2^y_q, y_q = (x - mq) c, e_p = 2^((x - mp) c).
struct Slope {
    float mq, a, b, mp, z, at_token;
    bool nothing;   // zeros all over the row
};
template <bool MASK> __device__ __forceinline__ Slope slope_of(const Sums &all, const Sums &q, float entropy, float logprob, const Upstream &up, int64_t b, int tok, const Temper &tp) {
    Slope s;
    const float g = up.logprobs && logprob > -INFINITY ? up.logprobs[b] : 0.f;   // (a log probability of -inf has no slope)
    const float z = MASK && up.logZ_valid ? up.logZ_valid[b] : 0.f, h = up.entropy ? up.entropy[b] : 0.f;
    s.nothing = tok < 0 || !(q.s != 0.f);
    const float over = tp.inv / q.s;
    s.mq = q.m;
    s.a = over * (z - g - h * (entropy - logf(q.s)));
    s.b = over * (-LN2F * h);
    s.mp = all.m;
    s.z = MASK ? z * tp.inv / all.s : 0.f;
    s.at_token = g * tp.inv;
    return s;
}
// Values of this lane's tokens from token v on, rounded to the nearest of their type, once.  What lies behind the row is left as it is.
__device__ __forceinline__ void put_group(float *row, int v, int V, const float (&d)[4]) {
    if (v + 4 <= V) {
        *(float4 *)(row + v) = {d[0], d[1], d[2], d[3]};
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; k++)
        if (v + k < V) row[v + k] = d[k];
}
__device__ __forceinline__ void put_group(uint16_t *row, int v, int V, const float (&d)[8]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; i++) r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){d[2 * i], d[2 * i + 1]}, bf16x2));
    if (v + 8 <= V) {
        *(u32x4 *)(row + v) = r;
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; k++)
        if (v + k < V) row[v + k] = (uint16_t)(r[k / 2] >> (16 * (k & 1)));
}
template <typename T, bool MASK, bool H>
__device__ __forceinline__ void put_tile(T *out, const MaskedTile<T> &mt, const Slope &s, int tile, int lane, int tok, int V, float c) {
    using G = TileGeom<T>;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const int v = tile * G::TILE + j * G::PER_LOAD + lane * G::EPL;
        float x[G::EPL], d[G::EPL];
        Elem<T>::unpack(mt.t.r[j], x);
        const uint32_t bits = MASK ? bits_fix<T>(mt.bits[j], lane) : 0u;
        const int mine = tok - v;   // the row's token, counted from this lane's first one
#pragma unroll
        for (int k = 0; k < G::EPL; k++) {
            const float y = (x[k] - s.mq) * c, e = fast_exp2(y);
            float g = e * (H ? fmaf(s.b, most(y, FAINT), s.a) : s.a);
            if (MASK) {
                g = (bits >> k) & 1u ? g : 0.f;
                g = fmaf(-s.z, fast_exp2((x[k] - s.mp) * c), g);
            }
            d[k] = mine == k ? g + s.at_token : g;
        }
        put_group(out, v, V, d);
    }
}
template <typename T> __device__ __forceinline__ void put_zeros(T *out, int first, int step, int lane, int V) {
    using G = TileGeom<T>;
    const float d[G::EPL] = {};
    for (int t = first; t * G::TILE < V; t += step)
#pragma unroll
        for (int j = 0; j < 4; j++) put_group(out, t * G::TILE + j * G::PER_LOAD + lane * G::EPL, V, d);
}
template <typename T, bool MASK, bool H>
__device__ __forceinline__ void put_row(T *out, const Row &row, const Row &mask, const Slope &s, int tok, int V, int first, int step, int lane, float c) {
    if (s.nothing) {
        put_zeros<T>(out, first, step, lane, V);
        return;
    }
    MaskedTile<T> now, next;
    now.template load<MASK>(row, mask, first, lane);
    for (int t = first; t * TileGeom<T>::TILE < V; t += step) {
        next.template load<MASK>(row, mask, t + step, lane);   // (read before this tile is written: out may be the logits themselves)
        put_tile<T, MASK, H>(out, now, s, t, lane, tok, V, c);
        now = next;
    }
}
// `parts` workgroups to a row; SHORT_ROWS rows to a workgroup where a row is one tile.
template <typename T, bool MASK, bool H, bool ONE>
__global__ __launch_bounds__(ONE ? SHORT_ROWS *WAVE : MOST_WAVES *WAVE) void gradient_kernel(const T *logits, int64_t row_stride, const int32_t *__restrict__ tokens,
                                                                                            const uint32_t *__restrict__ mask, int V, int n_words, int B, int parts,
                                                                                            T *d_logits, int64_t d_row_stride, const float *__restrict__ stats,
                                                                                            Upstream up, Temper tp) {
    const int lane = threadIdx.x & (WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), nw = blockDim.x / WAVE;
    const int64_t units = ONE ? B : (int64_t)B * parts;
    const int per = ONE ? SHORT_ROWS : 1;
    for (int64_t u = (int64_t)blockIdx.x * per + (ONE ? wave : 0); u < units; u += (int64_t)gridDim.x * per) {
        const int64_t b = ONE ? u : u / parts;
        const int part = ONE ? 0 : (int)(u - b * parts);
        const int tok = tokens ? tokens[b] : V;
        const float *st = stats + b * PPV_LOGPROB_STATS;
        const Sums all = {st[0], st[1], 0.f}, q = {st[2], st[3], 0.f};
        const Slope s = slope_of<MASK>(all, q, st[4], st[5], up, b, tok, tp);
        const Row row = row_of(logits + b * row_stride, V);
        put_row<T, MASK, H>(d_logits + b * d_row_stride, row, MASK ? mask_of(mask, b, n_words) : row, s, tok, V, ONE ? 0 : part * nw + wave,
                            ONE ? 1 : nw * parts, lane, tp.c);
    }
}

// Both: the sums, then the gradient from the row read again (from cache).
template <typename T, bool MASK, bool W, bool ONE>
__global__ __launch_bounds__(ONE ? SHORT_ROWS *WAVE : MOST_WAVES *WAVE) void score_gradient_kernel(const T *logits, int64_t row_stride, const int32_t *__restrict__ tokens,
                                                                                                  const uint32_t *__restrict__ mask, int V, int n_words, int B,
                                                                                                  T *d_logits, int64_t d_row_stride, Outputs out, Upstream up, Temper tp) {
    __shared__ RowSums sh;
    const int lane = threadIdx.x & (WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), nw = ONE ? 1 : blockDim.x / WAVE;
    const int per = ONE ? SHORT_ROWS : 1, first = ONE ? 0 : wave;
    for (int64_t b = (int64_t)blockIdx.x * per + (ONE ? wave : 0); b < B; b += (int64_t)gridDim.x * per) {
        const int tok = tokens ? tokens[b] : V;
        T *to = d_logits + b * d_row_stride;
        if (tok < 0) {   // left out
            if (lane == 0 && first == 0) put_values(out, b, {0.f, 0.f, 0.f});
            put_zeros<T>(to, first, nw, lane, V);
            continue;
        }
        const T *at = logits + b * row_stride;
        const Row row = row_of(at, V), mrow = MASK ? mask_of(mask, b, n_words) : row;
        float x = first == 0 ? logit_of(at, MASK ? mask + b * n_words : nullptr, tok, V) : 0.f;
        Sums all = no_sums(), valid = no_sums();
        take_row<T, MASK, true, W>(row, mrow, V, first, nw, lane, tp.c, all, valid);
        all = over_wave<W && !MASK>(all, tp.c);
        if (MASK) valid = over_wave<W>(valid, tp.c);
        if (!ONE) {
            if (lane == 0) {
                sh.all[wave] = all;
                if (MASK) sh.valid[wave] = valid;
                if (wave == 0) sh.x = x;   // (read before a wavefront may write there)
            }
            __syncthreads();
            x = sh.x;
            all = over_waves<W && !MASK>(sh.all, nw, lane, tp.c);
            if (MASK) valid = over_waves<W>(sh.valid, nw, lane, tp.c);
        }
        const Sums q = MASK ? valid : all;
        const RowValues v = row_values<MASK>(all, q, x, tp);
        if (lane == 0 && first == 0) put_values(out, b, v);
        const Slope s = slope_of<MASK>(all, q, v.entropy, v.logprob, up, b, tok, tp);
        put_row<T, MASK, W>(to, row, mrow, s, tok, V, first, nw, lane, tp.c);
        if (!ONE) __syncthreads();   // before LDS is used again
    }
}

// ------------------------------------------------------------------------------------------
// The most probable tokens.  A candidate's key orders by logit, and by token where logits are equal (the lower one first, -0 and +0 are
// equal): 32 bits of the logit above the 18 of the token's complement.  0: no candidate (not valid, or -inf).
constexpr int TOKEN_BITS = 18, KEY_BITS = 32 + TOKEN_BITS, DIGIT = 10, BINS = 1 << DIGIT;
constexpr uint32_t TOKEN_MASK = (1u << TOKEN_BITS) - 1u;
static_assert(PPV_MAX_VOCAB <= 1 << TOKEN_BITS && KEY_BITS % DIGIT == 0, "key layout");
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float logit_at(uint32_t order) {
    return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order);
}
__device__ __forceinline__ uint64_t key_of(float x, int v) {
    return x == -INFINITY ? 0ull : (uint64_t)order_of(x) << TOKEN_BITS | (TOKEN_MASK - (uint32_t)v);
}

struct TopShared {
    RowSums sums;
    uint32_t bin[BINS];
    uint64_t list[PPV_TOP_MAX];
    uint64_t prefix;
    uint32_t n, want;
    int settled;
};
// every candidate of the row, one lane and one token at a time: f(key)
template <typename T, bool MASK, typename F>
__device__ __forceinline__ void each_candidate(const Row &row, const Row &mask, int V, int first, int step, int lane, F f) {
    using G = TileGeom<T>;
    for (int t = first; t * G::TILE < V; t += step) {
        MaskedTile<T> mt;
        mt.template load<MASK>(row, mask, t, lane);
#pragma unroll
        for (int j = 0; j < 4; j++) {
            float x[G::EPL];
            const int v = t * G::TILE + j * G::PER_LOAD + lane * G::EPL;
            unpack_group<T, true>(mt.t.r[j], V - v, x);
            const uint32_t bits = MASK ? bits_fix<T>(mt.bits[j], lane) : 0xFFu;
#pragma unroll
            for (int k = 0; k < G::EPL; k++) {
                const uint64_t key = (bits >> k) & 1u ? key_of(x[k], v + k) : 0ull;
                if (key) f(key);
            }
        }
    }
}
// The k largest keys of a row into sh.list, in any order; sh.n: how many there are.  Digit by digit from the top: how many candidates
// have each value of the digit below the digits settled so far, and in which of them the k-th largest lies.  By all wavefronts.
template <typename T, bool MASK>
__device__ __forceinline__ void select_row(TopShared &sh, const Row &row, const Row &mask, int V, int k, int wave, int nw, int lane) {
    const int tid = wave * WAVE + lane;
    if (tid == 0) {
        sh.prefix = 0;
        sh.want = (uint32_t)k;
        sh.settled = 0;
        sh.n = 0;
    }
    int shift = KEY_BITS - DIGIT;
    for (;; shift -= DIGIT) {
        for (int i = tid; i < BINS; i += nw * WAVE) sh.bin[i] = 0;
        __syncthreads();
        const uint64_t prefix = sh.prefix;
        each_candidate<T, MASK>(row, mask, V, wave, nw, lane, [&](uint64_t key) __attribute__((always_inline)) {
            if ((key >> shift) >> DIGIT == prefix) atomicAdd(&sh.bin[(key >> shift) & (BINS - 1)], 1u);
        });
        __syncthreads();
        if (wave == 0) {   // from the largest digit down, a lane has BINS / WAVE of them
            constexpr int PER = BINS / WAVE;
            const int hi = BINS - 1 - lane * PER;
            uint32_t mine = 0;
            for (int i = 0; i < PER; i++) mine += sh.bin[hi - i];
            const uint32_t upto = wave_incl_scan(mine), want = sh.want;
            const uint64_t reached = __ballot(upto >= want);
            if (!reached) {   // fewer than k candidates (only the first digit can say so): all of them
                if (lane == 0) {
                    sh.prefix = 0;
                    sh.settled = 2;
                }
            } else if (lane == __ffsll((long long)reached) - 1) {
                uint32_t before = upto - mine;
                int i = 0;
                while (before + sh.bin[hi - i] < want) before += sh.bin[hi - i++];
                sh.prefix = prefix << DIGIT | (uint64_t)(hi - i);
                sh.want = want - before;
                sh.settled = sh.bin[hi - i] == want - before;   // the whole bin is wanted
            }
        }
        __syncthreads();
        if (sh.settled || shift == 0) break;
    }
    const uint64_t least = sh.settled == 2 ? 1ull : sh.prefix << shift;
    each_candidate<T, MASK>(row, mask, V, wave, nw, lane, [&](uint64_t key) __attribute__((always_inline)) {
        if (key >= least) {
            const uint32_t i = atomicAdd(&sh.n, 1u);
            if (i < PPV_TOP_MAX) sh.list[i] = key;   // (at most k of them)
        }
    });
    __syncthreads();
}

template <typename T, bool MASK, bool W>
__global__ __launch_bounds__(MOST_WAVES *WAVE) void top_kernel(const T *__restrict__ logits, int64_t row_stride, const int32_t *__restrict__ tokens,
                                                              const uint32_t *__restrict__ mask, int V, int n_words, int B, int k,
                                                              int32_t *__restrict__ top_ids, float *__restrict__ top_logprobs, Outputs out, Temper tp) {
    __shared__ TopShared sh;
    const int lane = threadIdx.x & (WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), nw = blockDim.x / WAVE;
    for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
        const int tok = tokens ? tokens[b] : V;
        int32_t *ids = top_ids + b * k;
        float *lps = top_logprobs + b * k;
        if (tok < 0) {   // left out
            if (threadIdx.x == 0) put_values(out, b, {0.f, 0.f, 0.f});
            for (int i = threadIdx.x; i < k; i += blockDim.x) {
                ids[i] = -1;
                lps[i] = -INFINITY;
            }
            continue;
        }
        const T *at = logits + b * row_stride;
        const Row row = row_of(at, V), mrow = MASK ? mask_of(mask, b, n_words) : row;
        const float x = logit_of(at, MASK ? mask + b * n_words : nullptr, tok, V);
        Sums q = no_sums(), valid = no_sums();
        take_row<T, MASK, !MASK, W>(row, mrow, V, wave, nw, lane, tp.c, q, valid);
        if (MASK) q = valid;
        q = over_wave<W>(q, tp.c);
        if (lane == 0) sh.sums.all[wave] = q;
        __syncthreads();
        q = over_waves<W>(sh.sums.all, nw, lane, tp.c);
        const RowValues v = row_values<false>(q, q, x, tp);
        if (threadIdx.x == 0) put_values(out, b, v);
        select_row<T, MASK>(sh, row, mrow, V, k, wave, nw, lane);
        const int n = (int)min(sh.n, (uint32_t)k);
        for (int i = threadIdx.x; i < k; i += blockDim.x) {   // a candidate's place: how many are larger
            if (i >= n) {
                ids[i] = -1;
                lps[i] = -INFINITY;
                continue;
            }
            const uint64_t key = sh.list[i];
            int place = 0;
            for (int j = 0; j < n; j++) place += sh.list[j] > key;
            ids[place] = (int32_t)(TOKEN_MASK - ((uint32_t)key & TOKEN_MASK));
            lps[place] = row_values<false>(q, q, logit_at((uint32_t)(key >> TOKEN_BITS)), tp).logprob;
        }
        __syncthreads();   // before LDS is used again
    }
}

// ------------------------------------------------------------------------------------------
// Host side.
struct Shape {
    unsigned grid, block;
    bool one;   // rows of one tile
};
int tiles_of(int V, ppv_dtype dt) {
    const int tile = dt == PPV_F32 ? TileGeom<float>::TILE : TileGeom<uint16_t>::TILE;
    return (V + tile - 1) / tile;
}
// Wavefronts per row: a power of two, at most one per tile.
int waves_of(int nt, int64_t rows) {
    const int cap = rows <= 256 ? 16 : (nt >= 48 || rows <= 512 ? 8 : 4);
    int nw = 1;
    while (nw < nt && nw * 2 <= cap) nw <<= 1;
    return nw;
}
unsigned groups_of(int64_t n) { return (unsigned)(n < (int64_t)MOST_GROUPS ? n : (int64_t)MOST_GROUPS); }
Shape shape_of(int V, ppv_dtype dt, int B) {
    const int nt = tiles_of(V, dt);
    if (nt == 1) return {groups_of(((int64_t)B + SHORT_ROWS - 1) / SHORT_ROWS), SHORT_ROWS * WAVE, true};
    return {groups_of(B), (unsigned)waves_of(nt, B) * WAVE, false};
}

ppv_status check_row_args(const void *logits, ppv_dtype dt, int64_t row_stride, int32_t B, int32_t V, float temperature, Temper *tp) {
    if (B < 0 || !temper_for(temperature, tp)) return PPV_EINVAL;
    return B == 0 ? PPV_OK : check_logits_args(logits, dt, row_stride, V);
}
// d_logits: rows like the logits', or the logits themselves; nothing in between, where one row's gradient would be written over another's logits.
ppv_status check_gradient_args(const void *logits, ppv_dtype dt, int64_t row_stride, int32_t B, int32_t V, const void *d_logits, int64_t d_row_stride) {
    const ppv_status st = check_logits_args(d_logits, dt, d_row_stride, V);
    if (st != PPV_OK) return st;
    if (d_logits == logits && d_row_stride == row_stride) return PPV_OK;
    const uint64_t e = dt == PPV_F32 ? 4 : 2, x = (uint64_t)(uintptr_t)logits, y = (uint64_t)(uintptr_t)d_logits;
    const uint64_t nx = ((uint64_t)(B - 1) * (uint64_t)row_stride + (uint64_t)V) * e, ny = ((uint64_t)(B - 1) * (uint64_t)d_row_stride + (uint64_t)V) * e;
    return x < y + ny && y < x + nx ? PPV_EINVAL : PPV_OK;
}

// CALL(type, masked or not, entropy or not) for what the call's arguments say
#define PPV_PICK(DT, MASK, ENTROPY, CALL)                   \
    do {                                                    \
        if ((DT) == PPV_F32) {                              \
            if (MASK) {                                     \
                if (ENTROPY) CALL(float, true, true);       \
                else CALL(float, true, false);              \
            } else {                                        \
                if (ENTROPY) CALL(float, false, true);      \
                else CALL(float, false, false);             \
            }                                               \
        } else {                                            \
            if (MASK) {                                     \
                if (ENTROPY) CALL(uint16_t, true, true);    \
                else CALL(uint16_t, true, false);           \
            } else {                                        \
                if (ENTROPY) CALL(uint16_t, false, true);   \
                else CALL(uint16_t, false, false);          \
            }                                               \
        }                                                   \
    } while (0)

}  // namespace

extern "C" ppv_status ppv_token_logprobs(const void *logits, ppv_dtype dt, int64_t row_stride, const uint32_t *mask, const int32_t *tokens,
                                         int32_t B, int32_t V, float *logprobs, float *logZ_valid, float *entropy, float *stats,
                                         float temperature, void *stream) {
    Temper tp;
    const ppv_status st = check_row_args(logits, dt, row_stride, B, V, temperature, &tp);
    if (st != PPV_OK || B == 0) return st;
    if ((logprobs && !tokens) || (!logprobs && !logZ_valid && !entropy && !stats) || ((uintptr_t)stats & 15u) != 0) return PPV_EINVAL;
    const Outputs out = {logprobs, logZ_valid, entropy, stats};
    const Shape sh = shape_of(V, dt, B);
    const int n_words = (V + 31) / 32;
#define PPV_SCORE(T, MASK, ENTROPY)                                                                                                     \
    do {                                                                                                                                \
        if (sh.one)                                                                                                                     \
            hipLaunchKernelGGL((score_kernel<T, MASK, ENTROPY, true>), dim3(sh.grid), dim3(sh.block), 0, (hipStream_t)stream,           \
                               (const T *)logits, row_stride, tokens, mask, V, n_words, B, out, tp);                                    \
        else                                                                                                                            \
            hipLaunchKernelGGL((score_kernel<T, MASK, ENTROPY, false>), dim3(sh.grid), dim3(sh.block), 0, (hipStream_t)stream,          \
                               (const T *)logits, row_stride, tokens, mask, V, n_words, B, out, tp);                                    \
    } while (0)
    PPV_PICK(dt, mask, entropy || stats, PPV_SCORE);
    PPV_HIP_TRY(hipGetLastError());
    return PPV_OK;
}

extern "C" ppv_status ppv_token_logprobs_backward(const void *logits, ppv_dtype dt, int64_t row_stride, const uint32_t *mask,
                                                  const int32_t *tokens, const float *stats, const float *d_logprobs,
                                                  const float *d_logZ_valid, const float *d_entropy, int32_t B, int32_t V, void *d_logits,
                                                  int64_t d_row_stride, float temperature, void *stream) {
    Temper tp;
    ppv_status st = check_row_args(logits, dt, row_stride, B, V, temperature, &tp);
    if (st != PPV_OK || B == 0) return st;
    if (!stats || ((uintptr_t)stats & 15u) != 0 || (d_logprobs && !tokens)) return PPV_EINVAL;
    st = check_gradient_args(logits, dt, row_stride, B, V, d_logits, d_row_stride);
    if (st != PPV_OK) return st;
    const Upstream up = {d_logprobs, d_logZ_valid, d_entropy};
    Shape sh = shape_of(V, dt, B);
    const int n_words = (V + 31) / 32, nt = tiles_of(V, dt);
    int parts = 1;
    while (!sh.one && (int64_t)B * parts < 512 && (int)(sh.block / WAVE) * parts * 2 <= nt) parts *= 2;
    if (!sh.one) sh.grid = groups_of((int64_t)B * parts);
#define PPV_GRADIENT(T, MASK, ENTROPY)                                                                                                  \
    do {                                                                                                                                \
        if (sh.one)                                                                                                                     \
            hipLaunchKernelGGL((gradient_kernel<T, MASK, ENTROPY, true>), dim3(sh.grid), dim3(sh.block), 0, (hipStream_t)stream,        \
                               (const T *)logits, row_stride, tokens, mask, V, n_words, B, 1, (T *)d_logits, d_row_stride, stats, up, tp); \
        else                                                                                                                            \
            hipLaunchKernelGGL((gradient_kernel<T, MASK, ENTROPY, false>), dim3(sh.grid), dim3(sh.block), 0, (hipStream_t)stream,       \
                               (const T *)logits, row_stride, tokens, mask, V, n_words, B, parts, (T *)d_logits, d_row_stride, stats, up, tp); \
    } while (0)
    PPV_PICK(dt, mask, d_entropy, PPV_GRADIENT);
    PPV_HIP_TRY(hipGetLastError());
    return PPV_OK;
}

extern "C" ppv_status ppv_token_logprobs_grad(const void *logits, ppv_dtype dt, int64_t row_stride, const uint32_t *mask, const int32_t *tokens,
                                              const float *d_logprobs, const float *d_logZ_valid, const float *d_entropy, int32_t B, int32_t V,
                                              float *logprobs, float *logZ_valid, float *entropy, void *d_logits, int64_t d_row_stride,
                                              float temperature, void *stream) {
    Temper tp;
    ppv_status st = check_row_args(logits, dt, row_stride, B, V, temperature, &tp);
    if (st != PPV_OK || B == 0) return st;
    if ((logprobs || d_logprobs) && !tokens) return PPV_EINVAL;
    st = check_gradient_args(logits, dt, row_stride, B, V, d_logits, d_row_stride);
    if (st != PPV_OK) return st;
    const Upstream up = {d_logprobs, d_logZ_valid, d_entropy};
    const Outputs out = {logprobs, logZ_valid, entropy, nullptr};
    const Shape sh = shape_of(V, dt, B);
    const int n_words = (V + 31) / 32;
#define PPV_SCORE_GRADIENT(T, MASK, ENTROPY)                                                                                            \
    do {                                                                                                                                \
        if (sh.one)                                                                                                                     \
            hipLaunchKernelGGL((score_gradient_kernel<T, MASK, ENTROPY, true>), dim3(sh.grid), dim3(sh.block), 0, (hipStream_t)stream,  \
                               (const T *)logits, row_stride, tokens, mask, V, n_words, B, (T *)d_logits, d_row_stride, out, up, tp);   \
        else                                                                                                                            \
            hipLaunchKernelGGL((score_gradient_kernel<T, MASK, ENTROPY, false>), dim3(sh.grid), dim3(sh.block), 0, (hipStream_t)stream, \
                               (const T *)logits, row_stride, tokens, mask, V, n_words, B, (T *)d_logits, d_row_stride, out, up, tp);   \
    } while (0)
    PPV_PICK(dt, mask, entropy || d_entropy, PPV_SCORE_GRADIENT);
    PPV_HIP_TRY(hipGetLastError());
    return PPV_OK;
}

extern "C" ppv_status ppv_top_logprobs(const void *logits, ppv_dtype dt, int64_t row_stride, const uint32_t *mask, const int32_t *tokens,
                                       int32_t B, int32_t V, int32_t k, int32_t *top_ids, float *top_logprobs, float *logprobs,
                                       float *entropy, float temperature, void *stream) {
    Temper tp;
    if (k < 1) return PPV_EINVAL;
    if (k > PPV_TOP_MAX) return PPV_ERANGE;
    const ppv_status st = check_row_args(logits, dt, row_stride, B, V, temperature, &tp);
    if (st != PPV_OK || B == 0) return st;
    if (!top_ids || !top_logprobs || (logprobs && !tokens)) return PPV_EINVAL;
    const Outputs out = {logprobs, nullptr, entropy, nullptr};
    const int n_words = (V + 31) / 32;
    const unsigned block = (unsigned)waves_of(tiles_of(V, dt), B) * WAVE;
#define PPV_TOP(T, MASK, ENTROPY)                                                                                                       \
    hipLaunchKernelGGL((top_kernel<T, MASK, ENTROPY>), dim3(groups_of(B)), dim3(block), 0, (hipStream_t)stream, (const T *)logits,      \
                       row_stride, tokens, mask, V, n_words, B, k, top_ids, top_logprobs, out, tp)
    PPV_PICK(dt, mask, entropy, PPV_TOP);
    PPV_HIP_TRY(hipGetLastError());
    return PPV_OK;
}
