// Log probabilities of given tokens, their gradient with respect to the logits, and the most probable tokens of a row: what a model
// gives to tokens that are there already, where the sampling kernels draw new ones.
//
// With l = logits / T, p = softmax(l) over all tokens, q = softmax(l) over the valid ones (q = p without a mask), t the row's token:
//   log q_t        = l_t - log sum_valid e^l
//   log Z_valid    = log sum_valid e^l - log sum e^l
//   entropy        = -sum q log q = log S - (sum y e^y) / S       with y = l - reference, S = sum e^y over the valid tokens
//   d_l            = d_logprob (1[v = t] - q) + d_logZ (q - p) - d_entropy q (log q + entropy),   d_logits = d_l / T
// A row is read once, by all lanes of its wavefronts, each with its own running reference and sums relative to it; the lanes' sums are
// brought to one reference at the end.  Sums are fp32.  A lane adds 16 or 32 terms a tile, 512 in all by the rules below (4,096
// where one wavefront is asked for): those of s are of one sign, those of w, each times its exponent, below 0 but for tokens above the reference.
#include <mutex>

#include "ppv_rows.h"
#include "ppv_split.h"

namespace {

constexpr int MOST_WAVES = 16;       // wavefronts per row and workgroup
constexpr int SHORT_ROWS = 4;        // rows of one tile: so many to a workgroup, a wavefront each
constexpr float LOWEST = -3.402823466e38f;
constexpr float FAINT = -1000.f;     // as an exponent of 2: a weight of 0

__device__ __forceinline__ float most(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float most(float a, float b, float c) {   // (without the instruction that quiets a NaN first)
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
template <int N> __device__ __forceinline__ float most_of(const float (&x)[N], float so_far) {
    float m = so_far;
#pragma unroll
    for (int i = 0; i < N; i += 2) m = most(m, x[i], x[i + 1]);
    return m;
}
__device__ __forceinline__ float uniform(float x) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x))); }

// ------------------------------------------------------------------------------------------
// Sums over tokens, in two forms.
//   Run    s = sum 2^(x c - r), w = sum of each of these times its exponent: one multiply-add and an exponential a token.  Any r gives the
//          same sums as long as they stay inside fp32, so a lane's r is the first group's largest token and is raised only where one
//          lies RAISE above it: a comparison a group.  (x c is not rounded before r is taken from it, and r is a reference of its own, no logit's.)
//          r is no lower than -FAR_OFF: a caller's stand-in for -inf (the type's lowest number, -1e30) weighs nothing, and the sum of
//          nothing else is 0.  Rows beyond FAR_OFF, to either side, are seen by that or by their largest token, and summed again in the
//          careful form.
//   Sums   s = sum 2^((x - m) c): the difference first, exact for an x within a factor of 2 of m; the reference is the largest token.
// An empty sum has a reference of LOWEST, which is finite: no difference below is that of two infinities.
constexpr float FAR_OFF = 134217728.f;   // 2^27: below it the rounding of r is at most four units of the exponent
constexpr float RAISE = 12.f;            // units of the exponent; entropies lose 12 * 2^-24 where a row's largest token comes late
constexpr float FAINT_SUM = 0.00390625f;       // 2^-8: valid tokens that weigh less than that against most lanes' references get one of their own ...
constexpr float LOST_SUM = 3.725290298461914e-9f;   // ... and 2^-28: those of one lane
struct Run {
    float r, s, w;
};
struct Sums {
    float m, s, w;
};
__device__ __forceinline__ Run no_run() { return {-FAR_OFF, 0.f, 0.f}; }
__device__ __forceinline__ Sums no_sums() { return {LOWEST, 0.f, 0.f}; }

// A lane's share of a row.
struct Tally {
    Run all;            // over all tokens (W without a mask: with w)
    float top, limit;   // the largest token; one above `limit` raises the reference
    Run valid;          // with a mask: the valid tokens relative to all.r as it was, or is ...
    Run few;            // ... and relative to a reference of their own
    bool seen;          // bits of the mask
};
__device__ __forceinline__ Tally no_tally() { return {no_run(), -INFINITY, LOWEST, no_run(), no_run(), false}; }
__device__ __forceinline__ void refer(float &s, float &w, float d) {   // to a reference that lies -d above
    const float f = fast_exp2(d);
    w = f * fmaf(d, s, w);
    s *= f;
}
__device__ __forceinline__ float reference_at(float top, float c) { return most(top * c, -FAR_OFF); }
// Sums of valid tokens are brought together relative to what the heaviest of them weighs: not to the highest reference, which may be one that
// the little there is lies far below, and by whose distance the others' exponents would be rounded.  (The sum of all has its reference's weight.)
__device__ __forceinline__ float weight_of(const Run &a, float r) { return r + (a.s != 0.f ? fast_log2(a.s) : 0.f); }
template <bool W> __device__ __forceinline__ Run both(const Run &a, const Run &b) {
    const float ra = a.s != 0.f ? a.r : LOWEST, rb = b.s != 0.f ? b.r : LOWEST, R = most(weight_of(a, ra), weight_of(b, rb));
    const float da = most(ra - R, FAINT), db = most(rb - R, FAINT), fa = fast_exp2(da), fb = fast_exp2(db);
    return {R, fa * a.s + fb * b.s, W ? fa * fmaf(da, a.s, a.w) + fb * fmaf(db, b.s, b.w) : 0.f};
}
// A lane's valid tokens of the tile at hand, relative to the reference of all
struct Weights {
    float s, w;
    bool some;   // bits of the mask
};
// The lane's reference is raised to its largest token where that lies above the limit (lanes whose does not: nothing changes).  IN: there are
// valid tokens relative to it.  A largest token of NaN, which one that signals among the others makes (quiet ones are passed over), counts as +inf.
template <bool MASK, bool IN> __device__ __forceinline__ void raise(Tally &a, Weights &in, float c, float step) {
    if (__ballot(MASK ? !(a.top <= a.limit) : a.top > a.limit) != 0ull) {
        const bool up = a.top > a.limit;
        const float r = up ? reference_at(a.top, c) : a.all.r, d = a.all.r - r;
        refer(a.all.s, a.all.w, d);
        if (IN) refer(in.s, in.w, d);
        a.all.r = r;
        a.limit = up ? a.top + step : a.limit;
        if (MASK) a.top = a.top != a.top ? INFINITY : a.top;
    }
}
template <int N, bool W> __device__ __forceinline__ void add(Run &a, const float (&x)[N], float c) {
#pragma unroll
    for (int i = 0; i < N; i++) {
        const float y = fmaf(x[i], c, -a.r), e = fast_exp2(y);
        a.s += e;
        if (W) a.w = fmaf(most(y, FAINT), e, a.w);   // (-inf: nothing, not a NaN)
    }
}
__device__ __forceinline__ uint32_t all_ones_if(uint32_t bits, int k) { return (uint32_t)__builtin_amdgcn_sbfe((int)bits, (uint32_t)k, 1u); }
__device__ __forceinline__ float if_bit(float x, uint32_t bits, int k) {
    const uint32_t m = all_ones_if(bits, k);
    return __uint_as_float((m & __float_as_uint(x)) | (~m & 0xFF800000u));   // x or -inf
}
// Valid tokens with a reference of their own
template <int N, bool W> __device__ __forceinline__ void take_few(Tally &a, const float (&x)[N], float c) {
    const float top = N == 1 ? x[0] : most_of<N>(x, -INFINITY);
    const bool up = fmaf(top, c, -a.few.r) > RAISE;   // (a limit, or the largest token so far, would take a register)
    if (__ballot(up) != 0ull) {
        const float r = up ? reference_at(top, c) : a.few.r;
        refer(a.few.s, a.few.w, a.few.r - r);
        a.few.r = r;
    }
    add<N, W>(a.few, x, c);
}
// A group of a lane's tokens, `bits`: the valid ones.  Where few lanes have any they are left to be summed by themselves (true); else they are
// summed with the exponentials that are there.
constexpr int FEW_LANES = 12;
template <int N, bool MASK, bool W> __device__ __forceinline__ bool take_group(Tally &a, Weights &in, const float (&x)[N], uint32_t bits, float c, float step) {
    a.top = most_of<N>(x, a.top);
    raise<MASK, MASK>(a, in, c, step);
    const int lanes = MASK ? __popcll(__ballot(bits != 0u)) : 0;
    if (lanes > FEW_LANES) {
#pragma unroll
        for (int i = 0; i < N; i++) {
            const float y = fmaf(x[i], c, -a.all.r), e = fast_exp2(y);
            a.all.s += e;
            const float v = __uint_as_float(__float_as_uint(e) & all_ones_if(bits, i));
            in.s += v;
            if (W) in.w = fmaf(most(y, FAINT), v, in.w);
        }
        in.some |= bits != 0u;
        return false;
    }
    add<N, W && !MASK>(a.all, x, c);
    return lanes != 0;
}
// The tile's valid tokens join those before.  True: the lane's weigh too little against its reference, with those before, and are to be summed by
// themselves.  That is so for all lanes where it is for most: where the model disagrees with a broad mask, the exponents of valid
// tokens would be rounded as coarsely as they lie below the others', and an entropy is their mean.  (Half of V = 20,000 fp32 valid and lower by
// 10 / 20 in the logits, entropies off by 4.2e-7 / 4.2e-7, root mean square, the plain form's 3.1e-7; by 9.8e-7 / 14.5e-7 where each lane
// decides for itself, at 2^-40.  us so / now: scores of 1,024 rows at V = 256k bf16 under prefixes' masks 92.6 / 91.6, under broad ones 104.2 /
// 101.3, 4,096 rows at V = 8k fp32 27.5 / 28.2; gradients of 64 rows at V = 32k 10.1 / 10.2, of 500 at V = 50k fp32 42.8 / 43.1.)
template <bool W> __device__ __forceinline__ bool join(Tally &a, const Weights &in) {
    const float d = a.valid.r - a.all.r;
    if (__ballot(a.valid.s != 0.f && d != 0.f) != 0ull) {   // references have been raised
        const Run before = a.valid;
        refer(a.valid.s, a.valid.w, d);
        const bool leave = a.valid.s < LOST_SUM && before.s != 0.f;
        if (__ballot(leave) != 0ull) {   // a sum that would weigh too little keeps the one it has, among the few.  (Others are rounded once by the distance.)
            const Run few = both<W>(before, a.few);
            a.few.r = leave ? few.r : a.few.r;
            a.few.s = leave ? few.s : a.few.s;
            a.few.w = leave ? few.w : a.few.w;
            a.valid.s = leave ? 0.f : a.valid.s;
            a.valid.w = leave ? 0.f : a.valid.w;
        }
    }
    a.valid.r = a.all.r;
    const float sum = a.valid.s + in.s;
    const uint64_t some = __ballot(in.some), enough = __ballot(sum >= FAINT_SUM) & some;
    const bool alone = in.some && sum < (2 * __popcll(enough) < __popcll(some) ? INFINITY : LOST_SUM);
    a.valid.s = alone ? a.valid.s : sum;
    if (W) a.valid.w += alone ? 0.f : in.w;
    return alone;
}

template <typename T> __device__ __forceinline__ int tiles_in(int V) { return (V + TileGeom<T>::TILE - 1) / TileGeom<T>::TILE; }

template <bool W, bool VALID> __device__ __forceinline__ Run over_lanes(const Run &a) {   // the wavefront's
    const float r = a.s != 0.f ? a.r : LOWEST, R = wave_max(VALID ? weight_of(a, r) : r), d = most(r - R, FAINT), f = fast_exp2(d);
    return {R, wave_sum(f * a.s), W ? wave_sum(f * fmaf(d, a.s, a.w)) : 0.f};
}
// relative to a logit that makes the sum about 1: weights are then no smaller against it than they are.  (Any number will do.  At temperatures
// near fp32's largest numbers that logit is outside them, or 1 / c infinite: the largest number, against which the sum is V at most.)
__device__ __forceinline__ Sums sums_of(const Run &a, float c) {
    if (!(a.s != 0.f)) return no_sums();
    const float m = __builtin_amdgcn_fmed3f((a.r + fast_log2(a.s)) * __builtin_amdgcn_rcpf(c), LOWEST, -LOWEST), d = fmaf(-m, c, a.r), f = fast_exp2(d);
    return {m, f * a.s, f * fmaf(d, a.s, a.w)};
}

// A tile of a row and, in each lane, a word of its mask.
template <typename T, bool MASK> struct MaskedTile {
    RawTile t;
    __device__ __forceinline__ void load(const Row &row, const uint32_t *mask, int tile, int lane, int V) {
        load_tile<T>(row, tile, lane, t);
        if (MASK) t.word = tile_word_raw<T>(mask, tile, lane, V);
    }
    // once it has come: bits behind the row's end are 0
    __device__ __forceinline__ void settle(int tile, int lane, int V) {
        if (MASK) t.word = tile_word_fix<T>(t.word, tile, lane, V);
    }
    __device__ __forceinline__ uint32_t valid(int j, int lane) const { return MASK ? lane_bits<T>(t.word, j, lane) : 0u; }
};
// Bits of the tokens of a group that starts with token v, read by themselves
template <typename T> __device__ __forceinline__ uint32_t bits_at(const uint32_t *mask, int v, int V) {
    return v < V ? (mask[v >> 5] >> (v & 31)) & ((1u << Elem<T>::EPL) - 1u) : 0u;
}
template <typename T, bool PAD> __device__ __forceinline__ void unpack_group(const u32x4 &r, int left, float (&x)[Elem<T>::EPL]) {
    unpack_fresh<T>(r, x);
    if (PAD) {
        asm volatile("" : "+v"(left));   // (compared here: ahead of the loop over tiles each token's comparison takes two scalar registers)
#pragma unroll
        for (int k = 0; k < Elem<T>::EPL; k++) x[k] = k < left ? x[k] : -INFINITY;
    }
}
// A tile with at most two valid tokens in each word of its mask, which is what an ordinary prefix has: those are asked for once more by
// themselves (from cache; they come while the tile is summed), a word's to a lane, and cost an exponential or two in all.
template <typename T> struct Gathered {
    float x[2];
    __device__ __forceinline__ void load(const Row &row, uint32_t w, int tile, int lane) {
        const uint32_t at = (uint32_t)tile * (TileGeom<T>::TILE * sizeof(T)) + (uint32_t)lane * (32 * sizeof(T)), w2 = w & (w - 1u);
        x[0] = load_at(row, w ? at + (uint32_t)__builtin_ctz(w) * (uint32_t)sizeof(T) : OUTSIDE);
        x[1] = load_at(row, w2 ? at + (uint32_t)__builtin_ctz(w2) * (uint32_t)sizeof(T) : OUTSIDE);
    }
    static constexpr uint32_t OUTSIDE = 0xFFFFFF00u;   // behind every row: nothing is read
    __device__ static __forceinline__ float load_at(const Row &row, uint32_t at) {
        if (sizeof(T) == 4) return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(row.buf, at, 0, 0));
        return __uint_as_float((uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(row.buf, at, 0, 0) << 16);
    }
};
template <typename T, bool MASK, bool W, bool PAD, bool FEW>
__device__ __forceinline__ void take_groups(const MaskedTile<T, MASK> &mt, int left, int lane, float c, float step, Tally &a) {
    constexpr int EPL = Elem<T>::EPL;
    Weights in = {0.f, 0.f, false};
    uint32_t left_over = 0u;   // the groups whose valid tokens are still to be summed
#pragma unroll
    for (int j = 0; j < 4; j++) {
        float x[EPL];
        unpack_group<T, PAD>(mt.t.r[j], left - j * TileGeom<T>::PER_LOAD, x);
        if (FEW) {
            a.top = most_of<EPL>(x, a.top);
            raise<true, false>(a, in, c, step);
            add<EPL, false>(a.all, x, c);
        } else {
            left_over |= take_group<EPL, MASK, W>(a, in, x, mt.valid(j, lane), c, step) ? 1u << j : 0u;
        }
        __builtin_amdgcn_sched_barrier(0);   // one group's tokens in registers at a time
    }
    if (!FEW && MASK) {
        const bool alone = join<W>(a, in);
        if (__ballot(alone) != 0ull || left_over != 0u) {
#pragma unroll 1
            for (int j = 0; j < 4; j++) {
                const bool it = (left_over >> j) & 1u;
                if (!it && __ballot(alone) == 0ull) continue;
                const u32x4 raw = j == 0 ? mt.t.r[0] : j == 1 ? mt.t.r[1] : j == 2 ? mt.t.r[2] : mt.t.r[3];
                const uint32_t valid = mt.valid(j, lane), bits = it || alone ? valid : 0u;   // (every lane takes part in the exchange)
                float x[EPL];
                unpack_group<T, PAD>(raw, left - j * TileGeom<T>::PER_LOAD, x);
#pragma unroll
                for (int i = 0; i < EPL; i++) x[i] = if_bit(x[i], bits, i);
                take_few<EPL, W>(a, x, c);
            }
        }
    }
}
template <typename T, bool MASK, bool W>
__device__ __forceinline__ void take_tile(const Row &row, const MaskedTile<T, MASK> &mt, int tile, int V, int lane, float c, float step, Tally &a) {
    const int left = tokens_left<T>(V, tile, lane);
    const bool whole = (tile + 1) * TileGeom<T>::TILE <= V;
    const uint32_t w = MASK ? mt.t.word : 0u, w2 = w & (w - 1u);
    if (MASK) a.seen |= w != 0u;
    if (MASK && __ballot((w2 & (w2 - 1u)) != 0u) == 0ull) {
        Gathered<T> g;
        g.load(row, w, tile, lane);
        if (whole) take_groups<T, MASK, W, false, true>(mt, left, lane, c, step, a);
        else take_groups<T, MASK, W, true, true>(mt, left, lane, c, step, a);
        if (__ballot(w != 0u) != 0ull) {
            const float x0[1] = {w ? g.x[0] : -INFINITY};
            take_few<1, W>(a, x0, c);
            if (__ballot(w2 != 0u) != 0ull) {
                const float x1[1] = {w2 ? g.x[1] : -INFINITY};
                take_few<1, W>(a, x1, c);
            }
        }
    } else {
        if (whole) take_groups<T, MASK, W, false, false>(mt, left, lane, c, step, a);
        else take_groups<T, MASK, W, true, false>(mt, left, lane, c, step, a);
    }
}
// The wavefront's tiles from its i-th on: the next one is on its way while one is summed.
template <typename T, bool MASK, bool W>
__device__ __forceinline__ void take_tiles(const Row &row, const uint32_t *mask, int V, const Share &share, int i, int lane, float c, float step, Tally &a) {
    if (i >= share.n) return;
    MaskedTile<T, MASK> now, next;
    now.load(row, mask, share.at(i), lane, V);
    for (; i < share.n; i++) {
        next.load(row, mask, i + 1 < share.n ? share.at(i + 1) : NO_TILE, lane, V);
        now.settle(share.at(i), lane, V);
        take_tile<T, MASK, W>(row, now, share.at(i), V, lane, c, step, a);
        now = next;
    }
}

// The careful form, token by token relative to the largest one so far.
template <int N> __device__ __forceinline__ void take_careful(Sums &a, const float (&x)[N], float c) {
    const float m = most(most_of<N>(x, a.m), LOWEST);
    refer(a.s, a.w, most((a.m - m) * c, FAINT));
    a.m = m;
#pragma unroll
    for (int i = 0; i < N; i++) {
        const float y = (x[i] - m) * c, e = fast_exp2(y);
        a.s += e;
        a.w = fmaf(most(y, FAINT), e, a.w);
    }
}
__device__ __forceinline__ Sums over_lanes(Sums a, float c) {
    const float m = wave_max(a.m);
    refer(a.s, a.w, most((a.m - m) * c, FAINT));
    return {m, wave_sum(a.s), wave_sum(a.w)};
}
template <typename T, bool MASK>
__device__ __forceinline__ void take_row_careful(const Row &row, const uint32_t *mask, int V, int wave, int nw, int lane, float c, Sums &all, Sums &valid) {
    constexpr int EPL = Elem<T>::EPL;
    all = valid = no_sums();
#pragma unroll 1
    for (int v = (wave * WAVE + lane) * EPL; v < V; v += nw * WAVE * EPL) {   // (as little code as it takes)
        float x[EPL];
        unpack_group<T, true>(__builtin_amdgcn_raw_buffer_load_b128(row.buf, (uint32_t)v * (uint32_t)sizeof(T), 0, 0), V - v, x);
        take_careful<EPL>(all, x, c);
        if (MASK) {
            const uint32_t bits = bits_at<T>(mask, v, V);
#pragma unroll
            for (int k = 0; k < EPL; k++) x[k] = if_bit(x[k], bits, k);
            take_careful<EPL>(valid, x, c);
        }
    }
    all = over_lanes(all, c);
    valid = over_lanes(valid, c);
}

// What a wavefront, a workgroup or several of them have found in their share of a row.
struct Part {
    Run all, valid;   // over all tokens, and over the valid ones (TWO: they are told apart)
    float top;        // the largest token
    uint32_t seen;    // 1: there were valid tokens
};
template <bool TWO, bool W> __device__ __forceinline__ Part over_lanes(const Part &p) {
    const bool some = TWO && __ballot(p.valid.s != 0.f) != 0ull;
    return {over_lanes<W && !TWO, false>(p.all), some ? over_lanes<W, true>(p.valid) : no_run(), wave_max(p.top),
            TWO && __ballot(p.seen != 0u) != 0ull ? 1u : 0u};
}
__device__ __forceinline__ Part no_part() { return {no_run(), no_run(), -INFINITY, 0u}; }

constexpr int NOT_COME = 2;
struct RowShared {
    Part part[MOST_WAVES];
    Part met;   // of all workgroups of a split row
    Sums careful_all[MOST_WAVES], careful_valid[MOST_WAVES];
    float x;    // the row's token's logit
    int mine;   // this workgroup finishes the row; NOT_COME: without all of the others' words
};
// A workgroup's wavefronts' tallies and the token's logit (`x`: known to wavefront 0), to every wavefront.  ONE: there is one.
template <bool TWO, bool W, bool ONE> __device__ __forceinline__ Part workgroup_part(RowShared &sh, const Tally &a, float &x, int wave, int nw, int lane) {
    const Run valid = !TWO ? no_run() : __ballot(a.few.s != 0.f) != 0ull ? both<W>(a.valid, a.few) : a.valid;
    Part p = over_lanes<TWO, W>({a.all, valid, a.top, a.seen ? 1u : 0u});
    if (ONE) return p;
    if (lane == 0) {
        sh.part[wave] = p;
        if (wave == 0) sh.x = x;   // (read before a wavefront may write there)
    }
    __syncthreads();
    x = sh.x;
    return over_lanes<TWO, W>(lane < nw ? sh.part[lane] : no_part());
}

// A split row's workgroups hand over their parts as words of the row's scratch, PART_WORDS each.  (by wavefront 0)
constexpr int PART_WORDS = 8;
static_assert(PPV_SPLIT_MAX_PARTS * PART_WORDS == 2 * WAVE, "two words a lane");
__device__ __forceinline__ void send_part(const Split &sp, const Part &p, int lane) {
    const float words[PART_WORDS] = {p.all.r, p.all.s, p.all.w, p.valid.r, p.valid.s, p.valid.w, p.top, __uint_as_float(p.seen)};
    float v = words[0];
#pragma unroll
    for (int i = 1; i < PART_WORDS; i++) v = lane == i ? words[i] : v;
    if (lane < PART_WORDS) send((Marked *)sp.row + sp.part * PART_WORDS + lane, v, sp.mark);
}
struct PartWords {
    Marked a, b;
};
__device__ __forceinline__ PartWords look_at_parts(const Split &sp, int lane) {   // (no lane without a word: conditions are registers)
    const Marked *at = (const Marked *)sp.row;
    const int n = sp.parts * PART_WORDS;
    return {shared_get(at + min(lane, n - 1)), shared_get(at + min(lane + WAVE, n - 1))};
}
// The parts of all workgroups, once they have arrived.  Words that do not come leave NaN.
template <bool TWO, bool W> __device__ __forceinline__ Part receive_parts(const Split &sp, PartWords w, int lane) {
    const bool come = wait_for(sp, [&]() __attribute__((always_inline)) { return has(w.a, sp.mark) && has(w.b, sp.mark); },
                               [&]() __attribute__((always_inline)) { w = look_at_parts(sp, lane); });
    Marked *at = (Marked *)sp.row;
    const int n = sp.parts * PART_WORDS;
    if (lane < n) shared_put(at + lane, (Marked)0);   // (for a graph, all of whose replays have one mark)
    if (lane + WAVE < n) shared_put(at + lane + WAVE, (Marked)0);
    float v[PART_WORDS];
#pragma unroll
    for (int i = 0; i < PART_WORDS; i++) {   // lane l: part l
        const int from = (lane & 7) * PART_WORDS + i;
        const float a = __shfl(value(w.a), from, WAVE), b = __shfl(value(w.b), from, WAVE);
        v[i] = lane < 8 ? a : b;
    }
    Part p = over_lanes<TWO, W>(lane < sp.parts ? Part{{v[0], v[1], v[2]}, {v[3], v[4], v[5]}, v[6], __float_as_uint(v[7])} : no_part());
    if (!come) p.all.s = p.valid.s = __uint_as_float(0x7FC00000u);
    return p;
}

struct RowSums {
    Sums all, q;   // over all tokens, and over the valid ones
};
// By every wavefront of the workgroup that has the row's part (ONE: the only one).  ONLY: the part is of the valid tokens alone, and so is
// the result.
template <typename T, bool MASK, bool ONE, bool ONLY = false>
__device__ __forceinline__ RowSums row_sums(RowShared &sh, const Row &row, const uint32_t *mask, int V, const Part &p, int wave, int nw, int lane, float c) {
    constexpr bool TWO = MASK && !ONLY;
    // (+inf or NaN at a token that is not valid has raised a reference over valid ones: they are summed again, relative to the largest of themselves)
    const bool far = TWO && p.top == INFINITY ? p.seen != 0u
                                              : fabsf(p.top) < INFINITY && (fabsf(p.top * c) >= FAR_OFF || (TWO && p.seen && p.valid.s == 0.f));
    RowSums r;
    if (__builtin_expect(__builtin_amdgcn_readfirstlane(far), 0)) {   // (the same for all wavefronts of the row)
        take_row_careful<T, MASK>(row, mask, V, wave, nw, lane, c, r.all, r.q);
        if (!ONE) {
            if (lane == 0) {
                sh.careful_all[wave] = r.all;
                sh.careful_valid[wave] = r.q;
            }
            __syncthreads();
            r.all = over_lanes(lane < nw ? sh.careful_all[lane] : no_sums(), c);
            r.q = over_lanes(lane < nw ? sh.careful_valid[lane] : no_sums(), c);
        }
        if (!MASK) r.q = r.all;
        return r;
    }
    r.all = sums_of(p.all, c);
    r.q = TWO ? sums_of(p.valid, c) : r.all;
    return r;
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
// (a - b) / T + more; the difference may be outside fp32 where this is not
__device__ __forceinline__ float over_t(float a, float b, const Temper &tp, float more) { return 2.f * fmaf(fmaf(-0.5f, b, 0.5f * a), tp.inv, 0.5f * more); }
// what the sums say.  Without mass (no valid token, or all at -inf): -inf, and an entropy of 0.
template <bool MASK> __device__ __forceinline__ RowValues row_values(const Sums &all, const Sums &q, float x, const Temper &tp, float log_s) {
    if (!(q.s != 0.f)) return {-INFINITY, -INFINITY, 0.f};
    const float logprob = over_t(x, q.m, tp, -log_s), logZ = MASK ? over_t(q.m, all.m, tp, log_s - logf(all.s)) : 0.f,
                entropy = fmaf(q.w / q.s, -LN2F, log_s);
    return {logprob > 0.f ? 0.f : logprob, logZ > 0.f ? 0.f : logZ, entropy < 0.f ? 0.f : entropy};   // (what rounding brings over the line)
}
template <bool MASK> __device__ __forceinline__ RowValues row_values(const Sums &all, const Sums &q, float x, const Temper &tp) {
    return row_values<MASK>(all, q, x, tp, logf(q.s));
}
static_assert(PPV_STATS_WORDS == PPV_LOGPROB_STATS, "one layout in both places");
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

template <bool SPLIT> __device__ __forceinline__ Split part_of(unsigned at_place, int shift) {
    if (!SPLIT) return {1, 0, nullptr, nullptr, 0u};
    return {1 << shift, (int)(at_place & ((1u << shift) - 1u)), nullptr, nullptr, 0u};
}
// Workgroup `group` of `groups` takes the place() -th piece of work.  Neighbouring workgroups start on the chip's eight dies in turn; a batch
// often has a period (a query's candidates, a sequence's positions), and rows of one kind, those near the root with long work on their
// masks, would all meet on one die.  So each die has a stretch of its own, and each round of its compute units starts at another place.
// (Scores under masks, every eighth row near the root, us in turn / so: 1,024 rows at V = 256k bf16 96.7 / 92.9 with four wavefronts, 4,096
// at V = 32k 53.1 / 49.2.)
constexpr unsigned DIES = 8, DIE_UNITS = 32;
__device__ __forceinline__ unsigned place(unsigned group, unsigned groups) {
    const unsigned die = group % DIES, each = groups / DIES, more = groups % DIES, mine = each + (die < more ? 1u : 0u);
    unsigned i = group / DIES;
    const unsigned round = i / DIE_UNITS;
    if ((round + 1u) * DIE_UNITS <= mine) i = round * DIE_UNITS + (i + 5u * round) % DIE_UNITS;
    return die * each + min(die, more) + i;
}

// ------------------------------------------------------------------------------------------
// Forward.  ONE: rows of one tile, a wavefront each; else a workgroup has a row, or (SPLIT) 1 << shift of them have.
template <typename T, bool MASK, bool W, bool ONE, bool SPLIT>
__global__ __launch_bounds__(ONE ? SHORT_ROWS *WAVE : MOST_WAVES *WAVE) void score_kernel(const T *__restrict__ logits, int64_t row_stride,
                                                                                         const int32_t *__restrict__ tokens, const uint32_t *__restrict__ mask,
                                                                                         int V, int n_words, int B, int shift, SplitScratch *scratch, uint32_t mark,
                                                                                         Outputs out, Temper tp) {
    __shared__ RowShared sh;
    const int lane = threadIdx.x & (WAVE - 1), wave = ONE ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), nw = ONE ? 1 : blockDim.x / WAVE;
    const unsigned at_place = place(blockIdx.x, gridDim.x);
    const int64_t b = ONE ? (int64_t)at_place * SHORT_ROWS + __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE) : at_place >> (SPLIT ? shift : 0);
    if (ONE && b >= B) return;
    Split sp = part_of<SPLIT>(at_place, shift);
    const int tok = tokens ? tokens[b] : V;
    if (tok < 0) {   // left out
        if (lane == 0 && wave == 0 && sp.part == 0) {
            put_values(out, b, {0.f, 0.f, 0.f});
            if (out.stats) put_stats(out.stats, b, {0.f, 0.f, 0.f}, {0.f, 0.f, 0.f}, {0.f, 0.f, 0.f});
        }
        return;
    }
    const T *at = logits + b * row_stride;
    const Row row = row_of(at, V);
    const uint32_t *mrow = MASK ? mask + b * n_words : nullptr;
    float x = wave == 0 ? logit_of(at, mrow, tok, V) : 0.f;
    Tally a = no_tally();
    take_tiles<T, MASK, W>(row, mrow, V, share_of(tiles_in<T>(V), sp.part * nw + wave, sp.parts * nw), 0, lane, tp.c, RAISE * __builtin_amdgcn_rcpf(tp.c), a);
    Part p = workgroup_part<MASK, W, ONE>(sh, a, x, wave, nw, lane);
    if (SPLIT) {
        if (wave == 0) {
            find_area<SPLIT>(sp, scratch, (int)b, mark);
            send_part(sp, p, lane);
            const PartWords w = look_at_parts(sp, lane);
            int last = 0;
            if (lane == 0) last = arrive(sp) ? 1 : 0;
            last = __builtin_amdgcn_readfirstlane(last);
            if (last) {
                p = receive_parts<MASK, W>(sp, w, lane);
                if (lane == 0) sh.met = p;
            }
            if (lane == 0) sh.mine = last;
        }
        __syncthreads();
        if (!sh.mine) return;
        p = sh.met;
    }
    const RowSums r = row_sums<T, MASK, ONE>(sh, row, mrow, V, p, wave, nw, lane, tp.c);
    if (lane == 0 && wave == 0) {
        const RowValues v = row_values<MASK>(r.all, r.q, x, tp);
        put_values(out, b, v);
        if (out.stats) put_stats(out.stats, b, r.all, r.q, v);
    }
}

// ------------------------------------------------------------------------------------------
// Gradient.
struct Upstream {
    const float *logprobs, *logZ_valid, *entropy;
};
// d_logits = e (a + b y) for valid tokens, less e_p z for all of them (a mask, and a slope of log Z), and `at_token` more at the row's token:
//   TOGETHER   y = x c - r, e = e_p = 2^y with r the reference of all tokens: one exponential a token.  For rows whose valid tokens weigh
//              enough against all: their exponents are as far below 0 then, and rounded as much more coarsely (2^-24 off for 2^-24 of the
//              weight is 1e-6, nothing to a gradient in bf16 but more than one in fp32 is rounded by: 2^-4)
//   else       y and e relative to the valid tokens' reference r, e_p = 2^(x c - rp)
// In rows beyond FAR_OFF, r and rp are logits, and y = (x - r) c.  So are they where b FAINT may be infinite, at temperatures below 1e-35: e is
// multiplied by y first then, which is 0 where e is.
constexpr float STEEP = 1e35f;
template <typename T> constexpr float TOGETHER_MOST = sizeof(T) == 4 ? 4.f : 24.f;
struct Slope {
    float r, a, b, rp, z, at_token;
    bool nothing;   // zeros all over the row
    bool far, together;
};
template <typename T, bool MASK> __device__ __forceinline__ Slope slope_of(const Sums &all, const Sums &q, float entropy, float logprob, const Upstream &up, int64_t b, int tok, const Temper &tp) {
    Slope s;
    const float g = up.logprobs && logprob > -INFINITY ? up.logprobs[b] : 0.f;   // (a log probability of -inf has no slope)
    const float z = MASK && up.logZ_valid ? up.logZ_valid[b] : 0.f, h = up.entropy ? up.entropy[b] : 0.f;
    const float over = 1.f / q.s, c = tp.c;   // (1 / T last: it may be one of fp32's subnormal numbers)
    s.nothing = __builtin_amdgcn_readfirstlane(tok < 0 || !(q.s != 0.f));
    s.a = over * (z - g - h * (entropy - logf(q.s))) * tp.inv;
    s.b = over * (-LN2F * h) * tp.inv;
    s.z = MASK && z != 0.f ? z / all.s * tp.inv : 0.f;
    s.far = __builtin_amdgcn_readfirstlane(!(fabsf(q.m * c) < FAR_OFF && fabsf(all.m * c) < FAR_OFF && fabsf(s.b) < STEEP));
    s.r = q.m;
    s.rp = all.m;
    s.together = false;
    if (!s.far) {   // relative to m c as it is rounded
        s.r = q.m * c;
        s.rp = all.m * c;
        float d = fmaf(-q.m, c, s.r);
        if (MASK) {
            s.together = __builtin_amdgcn_readfirstlane(s.z != 0.f && s.rp - s.r <= TOGETHER_MOST<T>);
            if (s.together) {
                d += s.rp - s.r;
                s.r = s.rp;
            }
            s.z *= fast_exp2(fmaf(-all.m, c, s.rp));
        }
        const float f = fast_exp2(d);
        s.a = f * fmaf(s.b, d, s.a);
        s.b *= f;
    }
    s.at_token = g * tp.inv;
    s.r = uniform(s.r), s.a = uniform(s.a), s.b = uniform(s.b), s.rp = uniform(s.rp), s.z = uniform(s.z), s.at_token = uniform(s.at_token);
    return s;
}
// Values of this lane's tokens from token v on, rounded to the nearest of their type, once.  What lies behind the row is left as it is.
__device__ __forceinline__ void put_group(float *row, int v, int V, const float (&d)[4]) {
    int left = V - v;
    asm volatile("" : "+v"(left));   // (see unpack_group)
    if (left >= 4) {
        typedef float f32x4 __attribute__((ext_vector_type(4)));
        __builtin_nontemporal_store((f32x4){d[0], d[1], d[2], d[3]}, (f32x4 *)(row + v));
    } else {
#pragma unroll
        for (int k = 0; k < 3; k++)
            if (k < left) row[v + k] = d[k];
    }
}
__device__ __forceinline__ void put_group(uint16_t *row, int v, int V, const float (&d)[8]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; i++) r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){d[2 * i], d[2 * i + 1]}, bf16x2));
    int left = V - v;
    asm volatile("" : "+v"(left));
    if (left >= 8) {
        __builtin_nontemporal_store(r, (u32x4 *)(row + v));
    } else {
#pragma unroll
        for (int k = 0; k < 7; k++)
            if (k < left) row[v + k] = (uint16_t)(r[k / 2] >> (16 * (k & 1)));
    }
}
template <bool FAR> __device__ __forceinline__ float exponent(float x, float r, float c) { return FAR ? (x - r) * c : fmaf(x, c, -r); }
template <typename T, bool MASK, bool H, bool FAR>
__device__ __forceinline__ void put_tile_as(T *out, const MaskedTile<T, MASK> &mt, const Slope &s, int tile, int lane, int tok, int V, float c) {
    using G = TileGeom<T>;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const int v = tile * G::TILE + j * G::PER_LOAD + lane * G::EPL;
        float x[G::EPL], d[G::EPL];
        unpack_fresh<T>(mt.t.r[j], x);
        const uint32_t bits = mt.valid(j, lane);
        const bool any = !MASK || __ballot(bits != 0u) != 0ull;
        if (MASK && !FAR && s.together) {
            if (any) {
#pragma unroll
                for (int k = 0; k < G::EPL; k++) {
                    const float y = fmaf(x[k], c, -s.r), e = fast_exp2(y), t = H ? fmaf(s.b, most(y, FAINT), s.a) : s.a;
                    d[k] = e * (__uint_as_float(__float_as_uint(t) & all_ones_if(bits, k)) - s.z);
                }
            } else {
#pragma unroll
                for (int k = 0; k < G::EPL; k++) d[k] = -s.z * fast_exp2(fmaf(x[k], c, -s.r));
            }
        } else {
#pragma unroll
            for (int k = 0; k < G::EPL; k++) d[k] = 0.f;
            if (any) {
#pragma unroll
                for (int k = 0; k < G::EPL; k++) {
                    const float y = exponent<FAR>(x[k], s.r, c), e = fast_exp2(y);
                    d[k] = !H ? e * s.a : FAR ? fmaf(e * most(y, FAINT), s.b, e * s.a) : e * fmaf(s.b, most(y, FAINT), s.a);
                    if (MASK) d[k] = __uint_as_float(__float_as_uint(d[k]) & all_ones_if(bits, k));
                }
            }
            if (MASK && s.z != 0.f) {
#pragma unroll
                for (int k = 0; k < G::EPL; k++) d[k] = fmaf(-s.z, fast_exp2(exponent<FAR>(x[k], s.rp, c)), d[k]);
            }
        }
        const int mine = tok - v;   // the row's token, counted from this lane's first one
        if (__ballot((uint32_t)mine < (uint32_t)G::EPL) != 0ull) {
#pragma unroll
            for (int k = 0; k < G::EPL; k++) d[k] = mine == k ? d[k] + s.at_token : d[k];
        }
        put_group(out, v, V, d);
        __builtin_amdgcn_sched_barrier(0);   // one group's tokens in registers at a time
    }
}
template <typename T, bool MASK, bool H>
__device__ __forceinline__ void put_tile(T *out, const MaskedTile<T, MASK> &mt, const Slope &s, int tile, int lane, int tok, int V, float c) {
    if (__builtin_expect(s.far, 0)) put_tile_as<T, MASK, H, true>(out, mt, s, tile, lane, tok, V, c);
    else put_tile_as<T, MASK, H, false>(out, mt, s, tile, lane, tok, V, c);
}
template <typename T> __device__ __forceinline__ void put_zeros(T *out, int first, int step, int lane, int V) {
    using G = TileGeom<T>;
    const float d[G::EPL] = {};
    for (int t = first; t * G::TILE < V; t += step)
#pragma unroll
        for (int j = 0; j < 4; j++) put_group(out, t * G::TILE + j * G::PER_LOAD + lane * G::EPL, V, d);
}
// The wavefront's tiles from the i-th on, which is asked for; each is read before another one is written: out may be the logits themselves.
template <typename T, bool MASK, bool H>
__device__ __forceinline__ void put_tiles(T *out, const Row &row, const uint32_t *mask, MaskedTile<T, MASK> &now, const Slope &s, int tok, int V, const Share &share, int i, int lane, float c) {
    MaskedTile<T, MASK> next;
    for (; i < share.n; i++) {
        next.load(row, mask, i + 1 < share.n ? share.at(i + 1) : NO_TILE, lane, V);
        now.settle(share.at(i), lane, V);
        put_tile<T, MASK, H>(out, now, s, share.at(i), lane, tok, V, c);
        now = next;
    }
}
// 1 << shift workgroups to a row; SHORT_ROWS rows to a workgroup where a row is one tile.
template <typename T, bool MASK, bool H, bool ONE>
__global__ __launch_bounds__(ONE ? SHORT_ROWS *WAVE : MOST_WAVES *WAVE) void gradient_kernel(const T *logits, int64_t row_stride, const int32_t *__restrict__ tokens,
                                                                                            const uint32_t *__restrict__ mask, int V, int n_words, int B, int shift,
                                                                                            T *d_logits, int64_t d_row_stride, const float *__restrict__ stats,
                                                                                            Upstream up, Temper tp) {
    const int lane = threadIdx.x & (WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), nw = blockDim.x / WAVE;
    const unsigned at_place = place(blockIdx.x, gridDim.x);
    const int64_t b = ONE ? (int64_t)at_place * SHORT_ROWS + wave : at_place >> shift;
    if (ONE && b >= B) return;
    const int first = ONE ? 0 : (int)(at_place & ((1u << shift) - 1u)) * nw + wave, of = ONE ? 1 : nw << shift;
    const int tok = tokens ? tokens[b] : V;
    T *to = d_logits + b * d_row_stride;
    if (tok < 0) {   // left out
        put_zeros(to, first, of, lane, V);
        return;
    }
    const Row row = row_of(logits + b * row_stride, V);
    const uint32_t *mrow = MASK ? mask + b * n_words : nullptr;
    const Share share = share_of(tiles_in<T>(V), first, of);
    MaskedTile<T, MASK> tile;   // (asked for ahead of what the slopes are made of)
    tile.load(row, mrow, share.n > 0 ? share.at(0) : NO_TILE, lane, V);
    const float *st = stats + b * PPV_LOGPROB_STATS;
    const Sums all = {st[0], st[1], 0.f}, q = {st[2], st[3], 0.f};
    const Slope s = slope_of<T, MASK>(all, q, st[4], st[5], up, b, tok, tp);
    if (s.nothing) put_zeros(to, first, of, lane, V);
    else put_tiles<T, MASK, H>(to, row, mrow, tile, s, tok, V, share, 0, lane, tp.c);
}

// Both: the sums, then the gradient.  A wavefront holds its first HELD tiles; MORE: it may have others, which are read again.  1 << shift
// workgroups may have a row: each takes all of its sums, which needs no word from another, and its part of the gradient.
template <typename T, bool MASK, bool W, bool ONE, int HELD, bool MORE>
__global__ __launch_bounds__(ONE ? SHORT_ROWS *WAVE : MOST_WAVES *WAVE) void score_gradient_kernel(const T *logits, int64_t row_stride, const int32_t *__restrict__ tokens,
                                                                                                  const uint32_t *__restrict__ mask, int V, int n_words, int B, int shift,
                                                                                                  T *d_logits, int64_t d_row_stride, Outputs out, Upstream up, Temper tp) {
    __shared__ RowShared sh;
    const int lane = threadIdx.x & (WAVE - 1), wave = ONE ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), nw = ONE ? 1 : blockDim.x / WAVE;
    const unsigned at_place = place(blockIdx.x, gridDim.x);
    const int64_t b = ONE ? (int64_t)at_place * SHORT_ROWS + __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE) : at_place >> shift;
    if (ONE && b >= B) return;
    const int part = ONE ? 0 : at_place & ((1 << shift) - 1);
    const int tok = tokens ? tokens[b] : V;
    T *to = d_logits + b * d_row_stride;
    if (tok < 0) {   // left out
        if (lane == 0 && wave == 0 && part == 0) put_values(out, b, {0.f, 0.f, 0.f});
        put_zeros(to, part * nw + wave, ONE ? 1 : nw << shift, lane, V);
        return;
    }
    const T *at = logits + b * row_stride;
    const Row row = row_of(at, V);
    const uint32_t *mrow = MASK ? mask + b * n_words : nullptr;
    const Share share = share_of(tiles_in<T>(V), wave, nw);
    MaskedTile<T, MASK> held[HELD];
#pragma unroll
    for (int i = 0; i < HELD; i++) held[i].load(row, mrow, i < share.n ? share.at(i) : NO_TILE, lane, V);
    float x = wave == 0 ? logit_of(at, mrow, tok, V) : 0.f;
    const float step = RAISE * __builtin_amdgcn_rcpf(tp.c);
    Tally a = no_tally();
#pragma unroll
    for (int i = 0; i < HELD; i++)
        if (i < share.n) {
            held[i].settle(share.at(i), lane, V);
            take_tile<T, MASK, W>(row, held[i], share.at(i), V, lane, tp.c, step, a);
        }
    if (MORE) take_tiles<T, MASK, W>(row, mrow, V, share, HELD, lane, tp.c, step, a);
    const Part p = workgroup_part<MASK, W, ONE>(sh, a, x, wave, nw, lane);
    const RowSums r = row_sums<T, MASK, ONE>(sh, row, mrow, V, p, wave, nw, lane, tp.c);
    const RowValues v = row_values<MASK>(r.all, r.q, x, tp);
    if (lane == 0 && wave == 0 && part == 0) put_values(out, b, v);
    const Slope s = slope_of<T, MASK>(r.all, r.q, v.entropy, v.logprob, up, b, tok, tp);
    if (s.nothing) {
        put_zeros(to, part * nw + wave, ONE ? 1 : nw << shift, lane, V);
        return;
    }
#pragma unroll
    for (int i = 0; i < HELD; i++)   // (four neighbouring wavefronts' tiles are one part's: those of the four SIMDs)
        if (i < share.n && (ONE || ((share.at(i) >> 2) & ((1 << shift) - 1)) == part)) put_tile<T, MASK, W>(to, held[i], s, share.at(i), lane, tok, V, tp.c);
    if (MORE) {
        MaskedTile<T, MASK> &tile = held[0];
        tile.load(row, mrow, HELD < share.n ? share.at(HELD) : NO_TILE, lane, V);
        put_tiles<T, MASK, W>(to, row, mrow, tile, s, tok, V, share, HELD, lane, tp.c);
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

constexpr int MOST_LISTED = 1024;   // candidates not below the bound that are sorted out in LDS
struct TopShared {
    RowShared row;
    union {   // one after the other, with a barrier between
        uint32_t best[MOST_WAVES * WAVE];   // each lane's largest token, and (up to two wavefronts) the largest of its other groups
        uint32_t bin[BINS];
        uint64_t list[MOST_LISTED];
    };
    uint64_t prefix;
    uint32_t n, want, bound;
    int settled;
};
// every candidate of the row, one lane and one token at a time: f(key)
template <typename T, bool MASK, typename F>
__device__ __forceinline__ void each_candidate(const Row &row, const uint32_t *mask, int V, int first, int step, int lane, F f) {
    using G = TileGeom<T>;
    for (int t = first; t * G::TILE < V; t += step) {
        MaskedTile<T, MASK> mt;
        mt.load(row, mask, t, lane, V);
        mt.settle(t, lane, V);
#pragma unroll
        for (int j = 0; j < 4; j++) {
            float x[G::EPL];
            const int v = t * G::TILE + j * G::PER_LOAD + lane * G::EPL;
            unpack_group<T, true>(mt.t.r[j], V - v, x);
            const uint32_t bits = MASK ? mt.valid(j, lane) : 0xFFu;
#pragma unroll
            for (int k = 0; k < G::EPL; k++) {
                const uint64_t key = (bits >> k) & 1u ? key_of(x[k], v + k) : 0ull;
                if (key) f(key);
            }
        }
    }
}
// The k largest keys of a row, or of the tiles first, first + of, ... of it, into sh.list, in any order; sh.n: how many there are.  Digit by
// digit from the top: how many candidates have each value of the digit below the digits settled so far, and in which of them the k-th
// largest lies.  By all wavefronts.
template <typename T, bool MASK>
__device__ __forceinline__ void select_row(TopShared &sh, const Row &row, const uint32_t *mask, int V, int k, int first, int of, int wave, int nw, int lane) {
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
        each_candidate<T, MASK>(row, mask, V, first, of, lane, [&](uint64_t key) __attribute__((always_inline)) {
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
    each_candidate<T, MASK>(row, mask, V, first, of, lane, [&](uint64_t key) __attribute__((always_inline)) {
        if (key >= least) {
            const uint32_t i = atomicAdd(&sh.n, 1u);
            if (i < MOST_LISTED) sh.list[i] = key;   // (k of them, or all there are)
        }
    });
    __syncthreads();
}

// What a lane remembers of its groups of tokens (16 bytes each) beside their sums: the group with the largest token, and the largest token
// of the others.
struct Best {
    float first, second;
    int at;   // 4 i + j: load j of the wavefront's i-th tile
    float third;   // HELD: the second largest group's place too, and the largest token of the others
    int at2;
};
template <typename T, bool MASK, bool W, bool PAD, bool HELD>
__device__ __forceinline__ void top_tile_as(const MaskedTile<T, MASK> &mt, int i, int left, int lane, float c, float step, Tally &a, Best &best) {
    constexpr int EPL = Elem<T>::EPL;
    Weights none;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const uint32_t bits = mt.valid(j, lane);
        if (MASK && __ballot(bits != 0u) == 0ull) continue;
        float x[EPL];
        unpack_group<T, PAD>(mt.t.r[j], left - j * TileGeom<T>::PER_LOAD, x);
        if (MASK) {
#pragma unroll
            for (int k = 0; k < EPL; k++) x[k] = if_bit(x[k], bits, k);
        }
        const float g = most_of<EPL>(x, -INFINITY);
        a.top = most(a.top, g);
        raise<false, false>(a, none, c, step);
        add<EPL, W>(a.all, x, c);
        if (HELD) {
            best.third = __builtin_amdgcn_fmed3f(best.second, best.third, g);
            best.at2 = g > best.first ? best.at : (g > best.second ? 4 * i + j : best.at2);
        }
        best.second = __builtin_amdgcn_fmed3f(best.first, best.second, g);   // (second <= first)
        best.at = g > best.first ? 4 * i + j : best.at;
        best.first = most(best.first, g);
        __builtin_amdgcn_sched_barrier(0);   // one group's tokens in registers at a time
    }
}
// A bound that at least k of the lanes' tokens `u` are not below: the k-th largest of them, or a little less; where SPARE is given, any that no
// more than k + SPARE are not below will do.  1 where there are fewer.  By one wavefront, bit by bit from the first in which they differ.
constexpr int BOUND_BITS = 12;
constexpr int FEW_ASKED = 20;   // up to so many candidates the bound is found from 64 tokens: a quarter more tokens reach it
template <int N, int BITS = BOUND_BITS, int SPARE = 0> __device__ __forceinline__ uint32_t bound_of(const uint32_t (&u)[N], int k) {
    uint32_t hi = 0u, lo = 0u;   // the largest, and the complement of the smallest that is one
    int some = 0;
#pragma unroll
    for (int i = 0; i < N; i++) {
        hi = max(hi, u[i]);
        lo = max(lo, u[i] ? ~u[i] : 0u);
        some += __popcll(__ballot(u[i] != 0u));
    }
    if (some < k) return 1u;
    hi = wave_max(hi);
    lo = ~wave_max(lo);
    if (hi == lo) return hi;
    const int first = 31 - __builtin_clz(hi ^ lo);
    uint32_t t = hi & ~((2u << first) - 1u);
    for (int bit = first; bit >= 0 && bit > first - BITS; bit--) {
        const uint32_t try_at = t | 1u << bit;
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; i++) n += __popcll(__ballot(u[i] >= try_at));
        if (n >= k) t = try_at;
        if (n >= k && n <= k + SPARE) break;
    }
    return t > 1u ? t : 1u;
}
// the bound as a logit: what is not below it is listed.  (1, no bound: anything but -inf)
__device__ __forceinline__ float bound_logit(uint32_t bound) { return bound > 1u ? most(logit_at(bound), LOWEST) : LOWEST; }
// The valid tokens of a group that are not below the bound
template <typename T>
__device__ __forceinline__ void list_group(TopShared &sh, const u32x4 &raw, uint32_t bits, int v, int V, float bound) {
    constexpr int EPL = Elem<T>::EPL;
    float x[EPL];
    uint32_t m = 0u;
    unpack_group<T, true>(raw, V - v, x);
#pragma unroll
    for (int k = 0; k < EPL; k++) m |= x[k] >= bound ? 1u << k : 0u;
    m &= bits;
    if (m) {
        uint32_t i = atomicAdd(&sh.n, (uint32_t)__builtin_popcount(m));
        do {   // (one, nearly always)
            const int k = __builtin_ctz(m);
            float at = x[0];
#pragma unroll
            for (int j = 1; j < EPL; j++) at = k == j ? x[j] : at;
            if (i < MOST_LISTED) sh.list[i] = key_of(at, v + k);
            i++;
            m &= m - 1u;
        } while (m);
    }
}
// Takes those of the n listed keys out that are not among the first k, but for a few and for ties of the last one's logit.  By one wavefront, in
// place.
constexpr int SPARE = 48, FEW_MORE = 12, MOST_ALIKE = 256;
template <int N> __device__ __forceinline__ int thin_out(TopShared &sh, int n, int k, int lane) {
    uint32_t u[N];
#pragma unroll
    for (int i = 0; i < N; i++) u[i] = i * WAVE + lane < n ? (uint32_t)(sh.list[i * WAVE + lane] >> TOKEN_BITS) : 0u;
    const uint32_t bound = bound_of<N, 32, FEW_MORE>(u, k);
    int kept = 0;
#pragma unroll 1
    for (int i = 0; i * WAVE < n; i++) {
        const uint64_t key = i * WAVE + lane < n ? sh.list[i * WAVE + lane] : 0ull;
        const bool keep = key >> TOKEN_BITS >= bound;
        const uint64_t who = __ballot(keep);
        if (keep) sh.list[kept + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u))] = key;
        kept += __popcll(who);
    }
    return kept;
}
// The same where it pays (placing n keys takes n^2 comparisons), by all wavefronts, with a barrier ahead; -1: more than `most` ties are left.
__device__ __forceinline__ int thinned_out(TopShared &sh, int n, int k, int most, int wave, int lane) {
    if (n <= k + SPARE) return n;
    if (wave == 0) {
        const int kept = n <= 4 * WAVE ? thin_out<4>(sh, n, k, lane) : thin_out<MOST_LISTED / WAVE>(sh, n, k, lane);
        if (lane == 0) sh.n = kept <= k + most ? kept : -1;
    }
    __syncthreads();
    return (int)sh.n;
}
// The row's first k of n listed keys, by all wavefronts: f(place, key) for each of them, in no order.  A key's place is how many are larger:
// a wavefront has every nw-th key, one to a lane, and counts for one after the other in as many comparisons as there are 64 keys; or, one or
// two wavefronts, each lane counts for its own, two at a time where there are more.  (73 of 364 bf16 tokens, 5,640 rows, one at a time 38.8 us,
// so 30.1, with the earlier end of the bound's search.)
template <typename F> __device__ __forceinline__ void each_place(const TopShared &sh, int n, int k, int wave, int nw, int lane, F f) {
    if (n <= nw * WAVE && nw <= 2) {
        const uint64_t key = wave * WAVE + lane < n ? sh.list[wave * WAVE + lane] : 0ull;
        int place = 0;
#pragma unroll 8
        for (int j = 0; j < n; j++) place += sh.list[j] > key;
        if (place < k && key) f(place, key);
        return;
    }
    if (nw <= 2) {
        for (int i = wave * WAVE + lane; i - lane < n; i += 2 * nw * WAVE) {   // (two keys a lane)
            const int i2 = i + nw * WAVE;
            const uint64_t key = i < n ? sh.list[i] : 0ull, key2 = i2 < n ? sh.list[i2] : 0ull;
            int place = 0, place2 = 0;
#pragma unroll 8
            for (int j = 0; j < n; j++) {
                const uint64_t other = sh.list[j];
                place += other > key;
                place2 += other > key2;
            }
            if (place < k && key) f(place, key);
            if (place2 < k && key2) f(place2, key2);
        }
        return;
    }
    for (int i0 = wave; i0 < n; i0 += nw * WAVE) {
        const int i = i0 + lane * nw, mine = min((n - i0 + nw - 1) / nw, WAVE);
        const uint64_t key = i < n ? sh.list[i] : 0ull;
        int place = 0;
        for (int j0 = 0; j0 < n; j0 += WAVE) {
            const uint64_t other = j0 + lane < n ? sh.list[j0 + lane] : 0ull;
            for (int l0 = 0; l0 < mine; l0 += 4) {   // (four that do not wait for one another)
#pragma unroll
                for (int l = l0; l < l0 + 4; l++) {
                    const uint64_t it = (uint64_t)lane_value((uint32_t)(key >> 32), l) << 32 | lane_value((uint32_t)key, l);
                    const int larger = __popcll(__ballot(other > it));
                    place += lane == l ? larger : 0;
                }
            }
        }
        if (place < k && key) f(place, key);
    }
}
// A split row's candidates lie behind its parts' sums, k to a part, two words each: the logit's order and the token's complement.
static_assert((sizeof(SplitRow) / sizeof(Marked) - PPV_SPLIT_MAX_PARTS * PART_WORDS) / 2 <= MOST_LISTED, "all parts' candidates are listed together");
int most_parts(int k) { return ((int)(sizeof(SplitRow) / sizeof(Marked)) - PPV_SPLIT_MAX_PARTS * PART_WORDS) / (2 * k); }
// HELD: a wavefront has as many tiles at most, and keeps them in registers.
template <typename T, bool MASK, bool W, bool SPLIT, int HELD>
__global__ __launch_bounds__(MOST_WAVES *WAVE) void top_kernel(const T *__restrict__ logits, int64_t row_stride, const int32_t *__restrict__ tokens,
                                                              const uint32_t *__restrict__ mask, int V, int n_words, int k, int shift, SplitScratch *scratch,
                                                              uint32_t mark, int32_t *__restrict__ top_ids, float *__restrict__ top_logprobs, Outputs out, Temper tp) {
    using G = TileGeom<T>;
    __shared__ TopShared sh;
    const int lane = threadIdx.x & (WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), nw = blockDim.x / WAVE;
    const unsigned at_place = place(blockIdx.x, gridDim.x);
    const int64_t b = at_place >> (SPLIT ? shift : 0);
    Split sp = part_of<SPLIT>(at_place, shift);
    const int tok = tokens ? tokens[b] : V;
    int32_t *ids = top_ids + b * k;
    float *lps = top_logprobs + b * k;
    if (tok < 0) {   // left out
        if (sp.part != 0) return;
        if (threadIdx.x == 0) put_values(out, b, {0.f, 0.f, 0.f});
        for (int i = threadIdx.x; i < k; i += blockDim.x) {
            ids[i] = -1;
            lps[i] = -INFINITY;
        }
        return;
    }
    const T *at = logits + b * row_stride;
    const Row row = row_of(at, V);
    const uint32_t *mrow = MASK ? mask + b * n_words : nullptr;
    float x = wave == 0 ? logit_of(at, mrow, tok, V) : 0.f;
    const int first = sp.part * nw + wave, of = sp.parts * nw;
    const Share share = share_of(tiles_in<T>(V), first, of);
    const float step = RAISE * __builtin_amdgcn_rcpf(tp.c);
    Tally a = no_tally();
    Best best = {-INFINITY, -INFINITY, 0, -INFINITY, 0};
    MaskedTile<T, MASK> held[HELD ? HELD : 1];
    auto take = [&](MaskedTile<T, MASK> &mt, int i) __attribute__((always_inline)) {
        const int tile = share.at(i), left = tokens_left<T>(V, tile, lane);
        mt.settle(tile, lane, V);
        if ((tile + 1) * G::TILE <= V) top_tile_as<T, MASK, W, false, HELD != 0>(mt, i, left, lane, tp.c, step, a, best);
        else top_tile_as<T, MASK, W, true, HELD != 0>(mt, i, left, lane, tp.c, step, a, best);
    };
    if (HELD) {
#pragma unroll
        for (int i = 0; i < HELD; i++) held[i].load(row, mrow, i < share.n ? share.at(i) : NO_TILE, lane, V);
#pragma unroll
        for (int i = 0; i < HELD; i++)
            if (i < share.n) take(held[i], i);
    } else {
        MaskedTile<T, MASK> now, next;
        now.load(row, mrow, share.n > 0 ? share.at(0) : NO_TILE, lane, V);
        for (int i = 0; i < share.n; i++) {
            next.load(row, mrow, i + 1 < share.n ? share.at(i + 1) : NO_TILE, lane, V);
            take(now, i);
            now = next;
        }
    }
    // the lanes' tokens that the bound is found from: 256 of them, or (one wavefront) 128
    const uint32_t mine = best.first == -INFINITY ? 0u : order_of(best.first), other = best.second == -INFINITY ? 0u : order_of(best.second);
    sh.best[wave * WAVE + lane] = mine;
    if (nw <= 2) sh.best[(nw + wave) * WAVE + lane] = other;
    if (threadIdx.x == 0) sh.n = 0;
    Part p = workgroup_part<false, W, false>(sh.row, a, x, wave, nw, lane);   // (a barrier behind what is above)
    if (wave == 0) {
        if (SPLIT) {
            find_area<SPLIT>(sp, scratch, (int)b, mark);
            send_part(sp, p, lane);
        }
        uint32_t u[4];
        const int have = nw <= 2 ? 2 * nw : nw;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            u[i] = 0u;
#pragma unroll
            for (int w = i; w < MOST_WAVES; w += 4) {   // (all asked for at once; what no wavefront has written is not looked at)
                const uint32_t v = sh.best[w * WAVE + lane];
                u[i] = max(u[i], w < have ? v : 0u);
            }
        }
        uint32_t bound;
        if (k <= FEW_ASKED) {
            const uint32_t one[1] = {max(max(u[0], u[1]), max(u[2], u[3]))};
            bound = bound_of(one, k);
        } else {
            bound = bound_of(u, k);
        }
        if (lane == 0) sh.bound = bound;
    }
    __syncthreads();
    const uint32_t bound = sh.bound;
    const float least = bound_logit(bound);
    auto token_of = [&](int i, int l) __attribute__((always_inline)) {   // the first one of lane l's group i
        return share.at(i >> 2) * G::TILE + (i & 3) * G::PER_LOAD + l * G::EPL;
    };
    const bool more = HELD ? best.third >= least : other >= bound;   // more groups than are remembered reach it
    const uint64_t lanes = __ballot(more);
    if (HELD) {
        auto list = [&](int group, bool listed) __attribute__((always_inline)) {
            if (__ballot(listed) == 0ull) return;
            u32x4 raw = held[0].t.r[0];
            uint32_t bits = MASK ? held[0].valid(0, lane) : 0xFFu;
#pragma unroll
            for (int g = 1; g < 4 * HELD; g++) {
                const bool it = group == g;
                const uint32_t its = MASK ? held[g / 4].valid(g % 4, lane) : 0u;
#pragma unroll
                for (int i = 0; i < 4; i++) raw[i] = it ? held[g / 4].t.r[g % 4][i] : raw[i];
                if (MASK) bits = it ? its : bits;
            }
            if (listed) list_group<T>(sh, raw, bits, token_of(group, lane), V, least);
        };
        list(best.at, mine >= bound && !more);
        list(best.at2, other >= bound && !more);
    }
    {
        auto look = [&](int i, int l) __attribute__((always_inline)) {
            const int v = token_of(i, l);
            list_group<T>(sh, __builtin_amdgcn_raw_buffer_load_b128(row.buf, (uint32_t)v * (uint32_t)sizeof(T), 0, 0),
                          MASK ? bits_at<T>(mrow, v, V) : 0xFFu, v, V, least);
        };
        if (!HELD && mine >= bound && !more) look(best.at, lane);
        // lanes with more than one such group: all of theirs are looked at again, one lane's by the whole wavefront or each its own
        if (__popcll(lanes) * ((share.n * 4 + WAVE - 1) / WAVE) > share.n * 4) {
            if (more)
                for (int i = 0; i < share.n * 4; i += 4) {   // (a tile's groups, asked for at once)
                    u32x4 raw[4];
                    uint32_t bits[4];
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const int v = token_of(i + j, lane);
                        raw[j] = __builtin_amdgcn_raw_buffer_load_b128(row.buf, (uint32_t)v * (uint32_t)sizeof(T), 0, 0);
                        bits[j] = MASK ? bits_at<T>(mrow, v, V) : 0xFFu;
                    }
#pragma unroll
                    for (int j = 0; j < 4; j++) list_group<T>(sh, raw[j], bits[j], token_of(i + j, lane), V, least);
                }
        } else {
            for (uint64_t rest = lanes; rest; rest &= rest - 1ull)
                for (int i = lane; i < share.n * 4; i += WAVE) look(i, __ffsll((long long)rest) - 1);
        }
    }
    __syncthreads();
    int n = (int)sh.n;
    __syncthreads();
    if (n <= MOST_LISTED) n = thinned_out(sh, n, k, MOST_ALIKE, wave, lane);
    if (n > MOST_LISTED || n < 0) {   // tokens that are too much alike
        __syncthreads();
        select_row<T, MASK>(sh, row, mrow, V, k, first, of, wave, nw, lane);
        n = (int)sh.n;
    }
    if (SPLIT) {
        find_area<SPLIT>(sp, scratch, (int)b, mark);
        Marked *words = (Marked *)sp.row + PPV_SPLIT_MAX_PARTS * PART_WORDS;
        each_place(sh, n, k, wave, nw, lane, [&](int place, uint64_t key) __attribute__((always_inline)) {
            Marked *w = words + 2 * (sp.part * k + place);
            send(w, __uint_as_float((uint32_t)(key >> TOKEN_BITS)), sp.mark);
            send(w + 1, __uint_as_float((uint32_t)key & TOKEN_MASK), sp.mark);
        });
        for (int i = n + (int)threadIdx.x; i < k; i += blockDim.x) {   // (the places that no candidate has)
            send(words + 2 * (sp.part * k + i), 0.f, sp.mark);
            send(words + 2 * (sp.part * k + i) + 1, 0.f, sp.mark);
        }
        __syncthreads();   // the workgroup's words are sent
        if (wave == 0) {
            const PartWords w = look_at_parts(sp, lane);
            int last = 0;
            if (lane == 0) last = arrive(sp) ? 1 : 0;
            last = __builtin_amdgcn_readfirstlane(last);
            if (last) {
                p = receive_parts<false, W>(sp, w, lane);
                if (lane == 0) {
                    sh.row.met = p;
                    sh.n = 0;
                }
            }
            if (lane == 0) sh.row.mine = last;
        }
        __syncthreads();
        if (!sh.row.mine) return;
        p = sh.row.met;
        const int most = sp.parts * k;
        for (int i0 = wave * WAVE; i0 < most; i0 += nw * WAVE) {   // (by whole wavefronts)
            const int i = min(i0 + lane, most - 1);
            Marked o, t;
            auto look_again = [&]() __attribute__((always_inline)) {
                o = shared_get(words + 2 * i);
                t = shared_get(words + 2 * i + 1);
            };
            look_again();
            const bool come = wait_for(sp, [&]() __attribute__((always_inline)) { return has(o, sp.mark) && has(t, sp.mark); }, look_again);
            shared_put(words + 2 * i, (Marked)0);
            shared_put(words + 2 * i + 1, (Marked)0);
            if (!come && lane == 0) sh.row.mine = NOT_COME;
            const uint64_t key = come ? (uint64_t)(uint32_t)o << TOKEN_BITS | ((uint32_t)t & TOKEN_MASK) : 0ull;
            if (i0 + lane < most && key) sh.list[atomicAdd(&sh.n, 1u)] = key;
        }
        __syncthreads();
        n = (int)sh.n;
        if (sh.row.mine == NOT_COME) {   // no candidates then, and a sum that is none
            n = 0;
            p.all.s = __uint_as_float(0x7FC00000u);
        }
        __syncthreads();
        n = thinned_out(sh, n, k, MOST_LISTED, wave, lane);
    }
    const RowSums r = row_sums<T, MASK, false, true>(sh.row, row, mrow, V, p, wave, nw, lane, tp.c);
    const float log_s = logf(r.q.s);
    each_place(sh, n, k, wave, nw, lane, [&](int place, uint64_t key) __attribute__((always_inline)) {
        ids[place] = (int32_t)(TOKEN_MASK - ((uint32_t)key & TOKEN_MASK));
        lps[place] = row_values<false>(r.q, r.q, logit_at((uint32_t)(key >> TOKEN_BITS)), tp, log_s).logprob;
    });
    for (int i = n + (int)threadIdx.x; i < k; i += blockDim.x) {
        ids[i] = -1;
        lps[i] = -INFINITY;
    }
    if (wave == nw - 1 && lane == 0) put_values(out, b, row_values<false>(r.q, r.q, x, tp, log_s));   // (it has had the fewest keys)
}

// ------------------------------------------------------------------------------------------
// Host side.
int tiles_of(int V, ppv_dtype dt) {
    const int tile = dt == PPV_F32 ? TileGeom<float>::TILE : TileGeom<uint16_t>::TILE;
    return (V + tile - 1) / tile;
}
// Wavefronts per row: a power of two.  A small batch is over when its longest row is, a large one when the chip's issue slots or the memory are
// through with all of them; each wavefront takes part in what follows the pass over a row.  us with 1 / 2 / 4 / 8 / 16: scores under
// prefixes' masks, bf16, V = 8k, 300 rows 8.9 / 7.3 / 5.9 / 5.8, 4,000 rows 19.8 / 18.8 / 19.4; V = 32k, 4,096 rows 54.7 (two) / 49.2 / 55.6 / 100;
// V = 256k, 1,024 rows 92.9 (four) / 92.7 / 107; fp32, V = 2,100 (three tiles), 4,000 rows 12.6 / 13.1 / 15.8.  Alternatives, V = 3,224 bf16,
// 4,000 rows 12.6 / 13.4, but 128 of them of V = 2,932, 3,408 rows 84.8 / 33.1; V = 8k 18.6 / 19.0 / 21.4; 300 rows 9.4 / 8.0 / 7.1 / 7.0.
int waves_of(int nt, int64_t rows, int k = 0) {   // k: alternatives; more than 64 of them are not bounded well by one wavefront's 128 maxima
    int cap = rows <= 256 ? 16 : (nt >= 48 || rows <= 512 ? 8 : 4);
    if (rows >= 2048 && nt <= 4) cap = nt <= 3 && k <= WAVE ? 1 : (k ? 2 : 4);
    if (const int v = ppv_tuning(PPV_TUNE_WAVES_PER_ROW)) cap = v;
    int nw = 1;
    while (nw < nt && nw * 2 <= cap) nw <<= 1;
    return nw;
}
// How many rows a launch takes: a grid has fewer than 2^32 threads.
constexpr int64_t MOST_ROWS = 1 << 21;
struct Shape {
    unsigned block;
    int per;    // rows to a workgroup
    bool one;   // rows of one tile
    unsigned groups(int64_t rows) const { return (unsigned)((rows + per - 1) / per); }
};
Shape shape_of(int V, ppv_dtype dt, int B) {
    const int nt = tiles_of(V, dt);
    if (nt == 1) return {SHORT_ROWS * WAVE, SHORT_ROWS, true};
    return {(unsigned)waves_of(nt, B) * WAVE, 1, false};
}
// The workgroups of a row (1 << shift), and where they meet.
struct Area {
    int shift;
    SplitScratch *scratch;
};
// More workgroups take more of the row off each and make more to hand over; batches beyond 256 workgroups leave no compute unit idle.
// us with 1 / 2 / 4 / 8 / 16, bf16 (masks as prefixes have them): scores, V = 32k, 16 rows 6.8 / 6.7 / 6.3 / 6.7 / 6.7, 128 rows 7.0 / 7.5 / 7.7;
// V = 64k, 1 row 9.7 / 8.3 / 6.7 / 6.4 / 6.6, 64 rows 10.0 / 8.6 / 7.6 / 8.5; V = 128k, 1 row 15.8 / 11.3 / 8.3 / 7.2 / 6.7, 32 rows 16.0 /
// 11.7 / 8.7 / 7.8 / 9.6, 128 rows 16.5 / 13.1 / 13.5; fp32 without masks, V = 50k, 128 rows 7.9 / 8.4 / 8.9.  Alternatives (20, without masks),
// V = 64k, 16 rows 10.3 / 10.4 / 10.2 / 14.9; V = 128k, 1 row 13.5 / 11.7 / 10.3 / 11.8, 64 rows 14.6 / 13.0 / 11.9 / 15.6, 128 rows 15.0 / 14.2 /
// 15.6; V = 256k, 32 rows 22.3 / 17.0 / 13.6 / 13.6; fp32, V = 50k, 128 rows 10.9 / 11.8 / 13.6.
// Every part's candidates are placed among those of all.  (V = 128k, 1 row, unsplit / in 4 / 8: 5 of them 12.8 / 9.4 / 8.4, 50
// of them 13.7 / 12.8 / 14.2, 128 of them 18.2 / 24.3; V = 64k 8.6 / 8.1 / 8.0, 10.3 / 11.8 / 17.1, 14.4 / 23.1.)
Area area_for(int V, ppv_dtype dt, int B, int k, int most, hipStream_t stream) {   // k: alternatives, 0 for scores
    const int nt = tiles_of(V, dt);
    int shift = 0;
    if (B <= PPV_SPLIT_MAX_ROWS) {
        if (const int v = ppv_tuning(PPV_TUNE_ROW_SPLIT)) {
            while ((2 << shift) <= v) shift++;
        } else {
            auto pays = [&](int parts) {
                if (B * parts > 256) return false;
                if (k) return parts <= 8 && parts * k <= 200 && (k <= 24 || nt >= 60) && nt / parts >= (B > 64 ? 28 : (k <= 8 ? 7 : 12));
                return nt / parts >= (B > 64 ? 16 : (parts >= 8 && B > 4 ? 6 : 4)) && (parts < 16 || B <= 4);
            };
            while ((2 << shift) <= PPV_SPLIT_MAX_PARTS && pays(2 << shift)) shift++;
        }
        while (shift && ((1 << shift) > most || 2 << shift > nt)) shift--;   // two tiles each
    }
    SplitScratch *scratch = shift ? ppv_split_scratch(stream, B) : nullptr;
    return {scratch ? shift : 0, scratch};
}
template <typename P> P *from_row(P *p, int64_t b, int64_t stride = 1) { return p ? p + b * stride : nullptr; }

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
#define PPV_LAUNCH(KERNEL, ...) hipLaunchKernelGGL(KERNEL, dim3(grid), dim3(block), 0, hs, __VA_ARGS__)

// A call's rows from row b on, `rows` of them.
struct Rows {
    int64_t at;
    int n, V, n_words;
    int64_t stride;
    const void *logits;
    const uint32_t *mask;
    const int32_t *tokens;
    hipStream_t stream;
    template <typename T> const T *logits_as() const { return (const T *)logits + at * stride; }
    const uint32_t *mask_rows() const { return from_row(mask, at, n_words); }
    const int32_t *token_rows() const { return from_row(tokens, at); }
};
Outputs from_row(const Outputs &o, int64_t b) {
    return {from_row(o.logprobs, b), from_row(o.logZ_valid, b), from_row(o.entropy, b), from_row(o.stats, b, PPV_LOGPROB_STATS)};
}
Upstream from_row(const Upstream &u, int64_t b) { return {from_row(u.logprobs, b), from_row(u.logZ_valid, b), from_row(u.entropy, b)}; }
// launch(rows) for all of a call's rows, MOST_ROWS at a time
template <typename F> ppv_status in_turns(Rows r, int B, F launch) {
    for (; r.at < B; r.at += MOST_ROWS) {
        r.n = (int)(B - r.at < MOST_ROWS ? B - r.at : MOST_ROWS);
        launch(r);
        PPV_HIP_TRY(hipGetLastError());
    }
    return PPV_OK;
}

template <typename T, bool MASK, bool W> void launch_score(const Rows &r, const Shape &sh, const Area &area, const Outputs &out, const Temper &tp) {
    const unsigned grid = sh.groups(r.n) << area.shift, block = sh.block;
    hipStream_t hs = r.stream;
#define PPV_SCORE(ONE, SPLIT)                                                                                                           \
    PPV_LAUNCH((score_kernel<T, MASK, W, ONE, SPLIT>), r.logits_as<T>(), r.stride, r.token_rows(), r.mask_rows(), r.V, r.n_words, r.n,    \
               area.shift, area.scratch, ppv_split_mark(area.shift), from_row(out, r.at), tp)
    if (sh.one) PPV_SCORE(true, false);
    else if (area.shift) PPV_SCORE(false, true);
    else PPV_SCORE(false, false);
#undef PPV_SCORE
}
template <typename T, bool MASK, bool H>
void launch_gradient(const Rows &r, const Shape &sh, int shift, void *d_logits, int64_t d_stride, const float *stats, const Upstream &up, const Temper &tp) {
    const unsigned grid = sh.one ? sh.groups(r.n) : (unsigned)r.n << shift, block = sh.block;
    hipStream_t hs = r.stream;
    T *d = (T *)d_logits + r.at * d_stride;
    const float *st = from_row(stats, r.at, PPV_LOGPROB_STATS);
    if (sh.one)
        PPV_LAUNCH((gradient_kernel<T, MASK, H, true>), r.logits_as<T>(), r.stride, r.token_rows(), r.mask_rows(), r.V, r.n_words, r.n, 0, d, d_stride, st, from_row(up, r.at), tp);
    else
        PPV_LAUNCH((gradient_kernel<T, MASK, H, false>), r.logits_as<T>(), r.stride, r.token_rows(), r.mask_rows(), r.V, r.n_words, r.n, shift, d, d_stride, st, from_row(up, r.at), tp);
}
// The tiles a wavefront holds of rows that it cannot hold whole: what is held is not read again, under masks four would not leave the registers
// that the sums take.  (us with none / two / three / four held by each of sixteen wavefronts, 600 rows: V = 100k fp32 134 / 124 / 115 / 108, masked
// 146 / 132 / 132, V = 160k 222 / 208 / 200 / 192, masked 231 / 216 / 220; 1,024 rows at V = 256k bf16 292 / 271 / 259 / 245, masked 304 / 280 / 289.)
constexpr int MOST_HELD = 4;
template <typename T, bool MASK, bool W>
void launch_score_gradient(const Rows &r, const Shape &sh, int held, int shift, void *d_logits, int64_t d_stride, const Outputs &out, const Upstream &up, const Temper &tp) {
    const unsigned grid = sh.groups(r.n) << shift, block = sh.block;
    hipStream_t hs = r.stream;
    T *d = (T *)d_logits + r.at * d_stride;
#define PPV_SCORE_GRADIENT(ONE, HELD, MORE)                                                                                                 \
    PPV_LAUNCH((score_gradient_kernel<T, MASK, W, ONE, HELD, MORE>), r.logits_as<T>(), r.stride, r.token_rows(), r.mask_rows(), r.V, r.n_words, \
               r.n, shift, d, d_stride, from_row(out, r.at), from_row(up, r.at), tp)
    if (sh.one) PPV_SCORE_GRADIENT(true, 1, false);
    else if (held > MOST_HELD) PPV_SCORE_GRADIENT(false, (MASK ? 2 : MOST_HELD), true);
    else if (held > 2) PPV_SCORE_GRADIENT(false, 4, false);
    else if (held > 1) PPV_SCORE_GRADIENT(false, 2, false);
    else PPV_SCORE_GRADIENT(false, 1, false);
#undef PPV_SCORE_GRADIENT
}
template <typename T, bool MASK, bool W>
void launch_top(const Rows &r, unsigned block, int held, const Area &area, int k, int32_t *top_ids, float *top_logprobs, const Outputs &out, const Temper &tp) {
    const unsigned grid = (unsigned)r.n << area.shift;
    hipStream_t hs = r.stream;
#define PPV_TOP(SPLIT, HELD)                                                                                                            \
    PPV_LAUNCH((top_kernel<T, MASK, W, SPLIT, HELD>), r.logits_as<T>(), r.stride, r.token_rows(), r.mask_rows(), r.V, r.n_words, k,      \
               area.shift, area.scratch, ppv_split_mark(area.shift), top_ids + r.at * k, top_logprobs + r.at * k, from_row(out, r.at), tp)
    if (area.shift && held <= 2) PPV_TOP(true, 2);
    else if (area.shift) PPV_TOP(true, 0);
    else if (held <= 2) PPV_TOP(false, 2);
    else PPV_TOP(false, 0);
#undef PPV_TOP
}

ppv_status score_call(const Rows &rows, ppv_dtype dt, int B, const Area &area, const Outputs &out, bool entropy, const Temper &tp) {
    const int nt = tiles_of(rows.V, dt);
    Shape sh = shape_of(rows.V, dt, B);
    if (area.shift) sh.block = (unsigned)waves_of((nt + (1 << area.shift) - 1) >> area.shift, (int64_t)B << area.shift) * WAVE;
    return in_turns(rows, B, [&](const Rows &r) {
#define PPV_CALL(T, MASK, W) launch_score<T, MASK, W>(r, sh, area, out, tp)
        PPV_PICK(dt, r.mask, entropy, PPV_CALL);
#undef PPV_CALL
    });
}
// Few rows of more tiles than this take two launches, the sums by several workgroups and then the gradient; others one, where a workgroup has all
// of a row's sums and reads again what it cannot hold (of more than 64 tiles).  Many parts gain most (up to 64 rows are split into four or more,
// then into two), and more under masks, whose sums take longer.  us in one launch / in two, masks as prefixes have them:
//   fp32    32 rows  56 tiles 10.4 / 10.3, 65 13.5 / 11.1, 250 59.8 / 21.4;  64 rows  60 tiles 11.2 / 12.4, 63 11.7 / 12.5, 65 14.5 / 13.9
//           96 rows  80 tiles 21.9 / 21.8, 88 24.7 / 23.0;  128 rows  98 tiles 30.0 / 31.6, 110 35.3 / 35.8, 128 42.3 / 40.8
//   masked  32 rows  36 tiles 12.7 / 12.5, 42 13.4 / 12.3;  64 rows  36 tiles 13.1 / 13.1, 39 13.3 / 13.2, 42 14.1 / 13.2, 98 32.1 / 21.0
//           96 rows  60 tiles 17.8 / 18.7, 63 19.4 / 19.1, 65 24.0 / 20.5;  128 rows  63 tiles 20.1 / 23.8, 65 26.3 / 25.2
//   bf16    32 rows  36 tiles 10.8 / 10.9, 40 11.5 / 11.0;  64 rows  36 tiles 11.2 / 11.6, 40 11.9 / 11.6, 128 42.1 / 24.6
//           96 rows  63 tiles 17.5 / 18.2, 65 21.5 / 19.8;  128 rows  80 tiles 28.3 / 28.7, 90 32.4 / 32.4, 105 38.0 / 36.5
//   masked   4 rows  27 tiles 12.5 / 12.5, broad masks 12.5 / 13.0, 29 13.6 / 12.3, 14.3 / 12.9;  64 rows  27 tiles 13.6 / 13.2, 13.6 / 13.6, 29 15.3 / 13.1
//           96 rows  32 tiles 16.3 / 14.5, 48 21.6 / 20.2 (fewer are not split);  128 rows  32 tiles 16.4 / 15.9, 40 18.2 / 20.3, 65 32.9 / 28.2
int tiles_of_one_launch(ppv_dtype dt, bool masked, int B) {
    const int rows = B <= 64 ? 0 : (B <= 96 ? 1 : 2);
    static constexpr int MOST[2][2][3] = {{{64, 84, 112}, {38, 62, 64}}, {{39, 64, 88}, {27, 31, 64}}};   // fp32, bf16; without a mask, under one
    return MOST[dt == PPV_F32 ? 0 : 1][masked ? 1 : 0][rows];
}
ppv_status gradient_call(const Rows &rows, ppv_dtype dt, int B, const float *stats, void *d_logits, int64_t d_stride, const Upstream &up, const Temper &tp) {
    Shape sh = shape_of(rows.V, dt, B);
    // No wavefront waits for another here.  us with 4 / 8 / 16 wavefronts, bf16: V = 32k, 64 rows 4.7 / 4.9 / 6.6, 2,048 rows 51.5 / 49.5 / 46.7;
    // V = 128k, 16 rows 4.6 / 5.2 / 7.5, 1,024 rows 104.4 / 102.6 / 99.1; V = 50k fp32, 128 rows 11.6 / 12.1 / 12.2, 400 rows 36.6 / 35.0 / 35.5.
    int nw = B < 256 ? 4 : (B < 512 ? 8 : MOST_WAVES);
    if (const int v = ppv_tuning(PPV_TUNE_WAVES_PER_ROW)) nw = v;
    while (nw > tiles_of(rows.V, dt) || (nw & (nw - 1))) nw--;
    if (!sh.one) sh.block = (unsigned)nw * WAVE;
    int shift = 0;
    while (!sh.one && (int64_t)B << shift < 512 && (int)(sh.block / WAVE) << (shift + 1) <= tiles_of(rows.V, dt)) shift++;
    return in_turns(rows, B, [&](const Rows &r) {
#define PPV_CALL(T, MASK, H) launch_gradient<T, MASK, H>(r, sh, shift, d_logits, d_stride, stats, up, tp)
        PPV_PICK(dt, r.mask, up.entropy, PPV_CALL);
#undef PPV_CALL
    });
}

}  // namespace

extern "C" ppv_status ppv_token_logprobs(const void *logits, ppv_dtype dt, int64_t row_stride, const uint32_t *mask, const int32_t *tokens,
                                         int32_t B, int32_t V, float *logprobs, float *logZ_valid, float *entropy, float *stats,
                                         float temperature, void *stream) {
    Temper tp;
    const ppv_status st = check_row_args(logits, dt, row_stride, B, V, temperature, &tp);
    if (st != PPV_OK || B == 0) return st;
    if ((logprobs && !tokens) || (!logprobs && !logZ_valid && !entropy && !stats) || ((uintptr_t)stats & 15u) != 0) return PPV_EINVAL;
    const Outputs out = {logprobs, logZ_valid, entropy, stats};
    const Area area = area_for(V, dt, B, 0, PPV_SPLIT_MAX_PARTS, (hipStream_t)stream);
    return score_call({0, 0, V, (V + 31) / 32, row_stride, logits, mask, tokens, (hipStream_t)stream}, dt, B, area, out, entropy || stats, tp);
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
    return gradient_call({0, 0, V, (V + 31) / 32, row_stride, logits, mask, tokens, (hipStream_t)stream}, dt, B, stats, d_logits, d_row_stride, up, tp);
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
    // (a row's workgroups each read what one of them would have written over)
    for (const float *o : {logprobs, logZ_valid, entropy})
        for (const float *u : {d_logprobs, d_logZ_valid, d_entropy})
            if (o && u && (uintptr_t)o < (uintptr_t)(u + B) && (uintptr_t)u < (uintptr_t)(o + B)) return PPV_EINVAL;
    const Upstream up = {d_logprobs, d_logZ_valid, d_entropy};
    Outputs out = {logprobs, logZ_valid, entropy, nullptr};
    const Rows rows = {0, 0, V, (V + 31) / 32, row_stride, logits, mask, tokens, (hipStream_t)stream};
    Shape sh = shape_of(V, dt, B);
    const int nt = tiles_of(V, dt);
    int nw = (int)sh.block / WAVE;
    while (!sh.one && nw < MOST_WAVES && nt > MOST_HELD * nw) nw *= 2;   // enough wavefronts to hold the row, if there are as many
    const int held = (nt + nw - 1) / nw;
    if (nt > tiles_of_one_launch(dt, mask != nullptr, B)) {
        const Area area = area_for(V, dt, B, 0, PPV_SPLIT_MAX_PARTS, (hipStream_t)stream);
        if (area.shift) {
            static std::mutex both;   // another thread's call on this stream does not come between the two launches
            const std::lock_guard<std::mutex> lock(both);
            out.stats = area.scratch->stats[0];
            st = score_call(rows, dt, B, area, out, entropy || d_entropy, tp);
            if (st != PPV_OK) return st;
            return gradient_call(rows, dt, B, out.stats, d_logits, d_row_stride, up, tp);
        }
    }
    // Two or four workgroups to a row of a small batch, up to one to a compute unit.  (us with one / two / four, V = 32k bf16 masked: 32 rows 11.2 / 10.0 /
    // 9.6, 64 rows 11.3 / 10.1 / 9.7, 128 rows 11.4 / 10.3 / 16.7; without masks 8.0 / 7.2 / 6.9, 8.3 / 7.5 / 7.2, 8.2 / 7.6 / 11.8; V = 50k fp32 64 rows
    // 11.1 / 9.9 / 9.7, 96 rows 11.2 / 10.2 / 18.2.)  They read the whole row: not where another one writes it.
    int shift = 0;
    while (!sh.one && held <= MOST_HELD && d_logits != logits && shift < 2 && nt >= 8 && (int64_t)B << (shift + 1) <= 256) shift++;
    if (!sh.one) sh.block = (unsigned)nw * WAVE;
    return in_turns(rows, B, [&](const Rows &r) {
#define PPV_CALL(T, MASK, W) launch_score_gradient<T, MASK, W>(r, sh, held, shift, d_logits, d_row_stride, out, up, tp)
        PPV_PICK(dt, mask, entropy || d_entropy, PPV_CALL);
#undef PPV_CALL
    });
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
    const Area area = area_for(V, dt, B, k, most_parts(k), (hipStream_t)stream);
    const int nt = (tiles_of(V, dt) + (1 << area.shift) - 1) >> area.shift, nw = waves_of(nt, (int64_t)B << area.shift, k), held = (nt + nw - 1) / nw;
    const unsigned block = (unsigned)nw * WAVE;
    return in_turns({0, 0, V, (V + 31) / 32, row_stride, logits, mask, tokens, (hipStream_t)stream}, B, [&](const Rows &r) {
#define PPV_CALL(T, MASK, W) launch_top<T, MASK, W>(r, block, held, area, k, top_ids, top_logprobs, out, tp)
        PPV_PICK(dt, mask, entropy, PPV_CALL);
#undef PPV_CALL
    });
}
