// A row of logits as the kernels of libppv_hip.so read it: its element types, the tiles it is loaded in, the bits of its mask, the
// temperature; and the host's checks of a call's logits.
#pragma once
#include <cmath>

#include "ppv_device.h"
#include "ppv_internal.h"

namespace {

constexpr float LN2F = 0.693147180559945309417f;

__device__ __forceinline__ float fast_exp2(float y) { return __builtin_amdgcn_exp2f(y); }  // v_exp_f32, 1 ulp
__device__ __forceinline__ float fast_log2(float y) { return __builtin_amdgcn_logf(y); }   // v_log_f32, 1 ulp (normal inputs)
// Temperature (Algorithm 1's input T): P = softmax(logits / T).  The division is folded into the constant of the
// exponentials, c = log2(e) / T, so that it costs nothing per token; differences of logits that enter a result
// as they are (a reference minus another) are multiplied by inv = 1 / T.  T = 1 gives c = log2(e), inv = 1.
struct Temper {
    float c;
    float inv;
    float guard;   // how far above an image tile's reference a logit may lie (REF_GUARD * T, see image_stats)
};

constexpr float REF_GUARD = 40.f;   // exp(40) * 2048 tokens is far inside fp32

// ------------------------------------------------------------------------------------------
// Tiles.  A tile is what one wavefront loads with four 16-byte loads per lane: 2048 bf16 or 1024
// fp32 tokens.  Load j of lane l holds the EPL consecutive tokens starting at
// tile*TILE + j*64*EPL + l*EPL, so token order inside a tile is (j, lane, k).
template <typename T> struct Elem;
template <> struct Elem<float> {
    static constexpr int EPL = 4;  // tokens per 16-byte load
    __device__ static __forceinline__ void unpack(const u32x4 &r, float x[4]) {
        x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y);
        x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
    }
};
template <> struct Elem<uint16_t> {  // bf16: widening to fp32 is exact
    static constexpr int EPL = 8;
    __device__ static __forceinline__ void unpack(const u32x4 &r, float x[8]) {
        x[0] = __uint_as_float(r.x << 16); x[1] = __uint_as_float(r.x & 0xFFFF0000u);
        x[2] = __uint_as_float(r.y << 16); x[3] = __uint_as_float(r.y & 0xFFFF0000u);
        x[4] = __uint_as_float(r.z << 16); x[5] = __uint_as_float(r.z & 0xFFFF0000u);
        x[6] = __uint_as_float(r.w << 16); x[7] = __uint_as_float(r.w & 0xFFFF0000u);
    }
};
// The same as unpack, with values that the compiler takes for new ones each time: what is unpacked is used at once and
// not kept in registers for another use of the tile (there is one in a rare case, and tiles are held packed).
template <typename T> __device__ __forceinline__ void unpack_fresh(const u32x4 &r, float x[Elem<T>::EPL]) {
    if (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; i++) x[i] = __uint_as_float(r[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            asm volatile("v_lshlrev_b32 %0, 16, %1" : "=v"(x[(2 * i) % Elem<T>::EPL]) : "v"(r[i]));
            asm volatile("v_and_b32 %0, %2, %1" : "=v"(x[(2 * i + 1) % Elem<T>::EPL]) : "v"(r[i]), "s"(0xFFFF0000u));
        }
    }
}
template <typename T> struct TileGeom {
    static constexpr int EPL = Elem<T>::EPL;
    static constexpr int PER_LOAD = WAVE * EPL;   // tokens covered by one load of the wave
    static constexpr int TILE = 4 * PER_LOAD;     // tokens per tile
    static constexpr int WORDS = TILE / 32;       // mask words per tile
    static constexpr int LANES_PER_WORD = 32 / EPL;
};

struct RawTile {
    u32x4 r[4];
    uint32_t word;   // image path: this lane's word of the tile's mask (requested together with the tile)
};

// A tile is requested with four unconditional 16-byte loads wherever it lies, also at the row's end and behind it; group_of puts
// -inf behind the end when the tile is used.  Nothing is conditional between request and use, so the compiler can
// count the loads in flight and wait for exactly the ones a use needs, and the ragged last tile is one like the others.
// One addition makes the four addresses (clamped into the row by comparisons, as here before, they took twelve).
template <typename T>
__device__ __forceinline__ void load_tile(const Row &row, int tile, int lane, RawTile &rt) {
    const uint32_t at = (uint32_t)tile * (4 * WAVE * 16u) + (uint32_t)lane * 16u;
#pragma unroll
    for (int j = 0; j < 4; j++) rt.r[j] = __builtin_amdgcn_raw_buffer_load_b128(row.buf, at + j * (WAVE * 16u), 0, 2 /* non-temporal */);
}
constexpr int NO_TILE = 1 << 18;   // behind every row: a request that reads nothing
// The tile's tokens that lie inside the row, counted from this lane's first one (PAD: what is behind the row's end counts
// as -inf; only the row's last tile has any of that).
template <typename T> __device__ __forceinline__ int tokens_left(int V, int tile, int lane) {
    return V - tile * TileGeom<T>::TILE - lane * TileGeom<T>::EPL;
}
// group j of a tile, unpacked
template <typename T, bool PAD> __device__ __forceinline__ void group_of(const RawTile &rt, int j, int left, float x[TileGeom<T>::EPL]) {
    unpack_fresh<T>(rt.r[j], x);
    if (PAD) {
        int in = left - j * TileGeom<T>::PER_LOAD;
        asm("" : "+v"(in));   // (or the compiler compares `left` with a constant for each token, each in a register of its own)
#pragma unroll
        for (int k = 0; k < TileGeom<T>::EPL; k++) x[k] = k < in ? x[k] : -INFINITY;
    }
}

// word wi of a V-bit image, with bits at positions >= V cleared (0 beyond the image), in two parts: the load, unconditional
// (clamped index: a conditional load would make later waits conservative), and what is done to the word once it is
// used (at the load it would wait for it, and for every tile asked for before).
__device__ __forceinline__ uint32_t image_word_raw(const uint32_t *__restrict__ image, int wi, int V) {
    const int last = (V + 31) / 32 - 1;
    return image[wi < last ? wi : last];
}
__device__ __forceinline__ uint32_t image_word_fix(uint32_t w, int wi, int V) {
    const int last = (V + 31) / 32 - 1;
    if (wi == last && (V & 31)) w &= (1u << (V & 31)) - 1u;
    return wi <= last ? w : 0u;
}
__device__ __forceinline__ uint32_t image_word(const uint32_t *__restrict__ image, int wi, int V) {
    return image_word_fix(image_word_raw(image, wi, V), wi, V);
}
// the tile's mask word for this lane (lane l < WORDS holds word l of the tile), in the same two parts
template <typename T> __device__ __forceinline__ uint32_t tile_word_raw(const uint32_t *__restrict__ image, int tile, int lane, int V) {
    using G = TileGeom<T>;
    return image_word_raw(image, tile * G::WORDS + (lane < G::WORDS ? lane : 0), V);
}
template <typename T> __device__ __forceinline__ uint32_t tile_word_fix(uint32_t w, int tile, int lane, int V) {
    using G = TileGeom<T>;
    return lane < G::WORDS ? image_word_fix(w, tile * G::WORDS + lane, V) : 0u;
}
template <typename T>
__device__ __forceinline__ uint32_t tile_mask_word(const uint32_t *__restrict__ image, int tile, int lane, int V) {
    return tile_word_fix<T>(tile_word_raw<T>(image, tile, lane, V), tile, lane, V);
}

// mask bits of this lane's EPL tokens of load j, from the tile's mask words (lane l < WORDS holds word l)
template <typename T> __device__ __forceinline__ uint32_t lane_bits(uint32_t tile_word, int j, int lane) {
    using G = TileGeom<T>;
    uint32_t w = (uint32_t)__shfl((int)tile_word, j * (G::WORDS / 4) + lane / G::LANES_PER_WORD, WAVE);
    return (w >> ((lane % G::LANES_PER_WORD) * G::EPL)) & ((1u << G::EPL) - 1u);
}

// A wavefront's share of a row: of `nw` wavefronts number `wave` has the tiles wave, wave + nw, ...  It takes them from a place
// on that the workgroup's number sets, and the last one, which may be ragged, last.  (Rows that are started together are
// otherwise read in step, and what is asked for at one time lies at the same place of a thousand rows: us per call, in
// step and like this, ppv_sample_next, 1,024 rows, V = 256k bf16 96.2 / 88.4, V = 128k 48.8 / 47.1; the decoding loop, 2,048
// rows at V = 32k, 547.7 / 541.2.  The sixteen places in the order of their bits reversed: neighbours start far apart.)
struct Share {
    int wave, nw, n, turn;   // n: tiles
    __device__ __forceinline__ int first() const { return wave + turn * nw; }
    __device__ __forceinline__ int at(int i) const {   // the i-th tile it takes
        int q = i + turn;
        q = q >= n - 1 ? q - (n - 1) : q;
        return wave + (i < n - 1 ? q : i) * nw;
    }
};
// `wave_v`: the wavefront's number among all that share the row, over all its workgroups
__device__ __forceinline__ Share share_of(int nt, int wave_v, int nw) {
    const int wave = __builtin_amdgcn_readfirstlane(wave_v);   // scalar: loop control stays uniform
    Share s = {wave, nw, 0, 0};
    const int up = nt - wave + nw - 1;
    if ((nw & (nw - 1)) == 0) s.n = up >> __builtin_ctz((unsigned)nw);   // (a division is a hundred cycles before the first load)
    else for (int x = up; x >= nw; x -= nw) s.n++;
    // (where a row has sixteen wavefronts it is nearly alone on its compute unit, and the numbers would only be waited for:
    // constrained_sample, 128 rows at V = 50,265 fp32, 11.0 us without, 11.8 with a turn)
    if ((nw <= 8 || (nw & (nw - 1)) != 0) && s.n > 2) s.turn = (int)((__brev(blockIdx.x) >> 28) * (uint32_t)(s.n - 1) >> 4);
    return s;
}

// T > 0 and finite, or the call is refused; the constants the kernels take (see Temper)
bool temper_for(float temperature, Temper *tp) {
    if (!(temperature > 0.f) || !std::isfinite(temperature)) return false;
    tp->c = (float)(1.44269504088896340736 / (double)temperature);   // log2(e) / T
    tp->inv = (float)(1.0 / (double)temperature);
    tp->guard = REF_GUARD * temperature;
    return std::isfinite(tp->c) && tp->c > 0.f;
}

ppv_status check_logits_args(const void *logits, ppv_dtype dt, int64_t row_stride, int32_t V) {
    if (!logits || V <= 0 || row_stride < V) return PPV_EINVAL;
    if (dt != PPV_F32 && dt != PPV_BF16) return PPV_EINVAL;
    const int64_t per16 = (dt == PPV_F32) ? 4 : 8;
    if (row_stride % per16 != 0 || ((uintptr_t)logits & 15u) != 0) return PPV_EINVAL;
    if (V > PPV_MAX_VOCAB) return PPV_ERANGE;
    return PPV_OK;
}

}  // namespace
