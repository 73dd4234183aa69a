// The cache of a serving loop (llla_cache of the C ABI): one problem as validated by the host, and the 8-bit format on the device.
//
// A block of 64 slots of a (sequence, head) shares one power of two: row = code * 2^e.  A power of two because the products are then exact
// (codes times it are bf16 and f16 numbers), a row goes from one block to another by a shift, and nothing is lost for it in e4m3, whose
// relative precision does not depend on the factor (int8 loses half a bit on average).
#pragma once

#include "llla_common.hpp"

namespace llla {

constexpr int CACHE_BLOCK = LLLA_CACHE_BLOCK;
constexpr int EXP_LEAST = -120;          // a block of zeros, or of values below it
constexpr int EXP_NAN = -128;            // a block that was given a value that is not finite

struct AppendProblem {
    llla_cache c;
    const void *k, *v;
    llla_strides sk, sv;
    int n;
    llla_dtype in;
    const int32_t *seqlens, *new_lens, *first_pos;
    hipStream_t stream;
};
hipError_t cache_append(const AppendProblem &p);

struct DecodeQ8Problem {
    llla_cache c;
    const void *q;
    void *o;
    const int32_t *seqlens;
    int H;
    llla_dtype in, out;
    float lambda, scale;
    void *ws;
    size_t ws_bytes;
    hipStream_t stream;
};
size_t decode_q8_workspace_bytes(int B, int H, int L_max, int d);
hipError_t decode_q8(const DecodeQ8Problem &p);

struct ScoresProblem {
    llla_cache c;
    const void *Q;
    llla_strides sq;
    const int32_t *seqlens;
    int H, nq;
    llla_dtype in;
    float scale;
    void *ws;
    hipStream_t stream;
};
size_t cache_scores_workspace_bytes(const llla_cache &c, int H, int nq, llla_dtype in);
hipError_t cache_scores(const ScoresProblem &p);

struct EvictProblem {
    llla_cache c, into;
    bool in_place;
    const int32_t *seqlens;
    int keep, sinks, recent;
    int32_t *lens, *index;
    void *ws;
    hipStream_t stream;
};
size_t cache_evict_workspace_bytes(const llla_cache &c, int keep);
hipError_t cache_evict(const EvictProblem &p);

__host__ __device__ inline int cache_blocks(int L_max) { return (L_max + CACHE_BLOCK - 1) / CACHE_BLOCK; }
__device__ inline int cache_length(const int32_t *seqlens, int b, int L_max) { return seqlens ? min(max(seqlens[b], 0), L_max) : L_max; }

// ---- the two formats ----------------------------------------------------------------------------------------------------------
struct Int8Code {
    static constexpr int POWER = 7;                        // largest value = FRACTION * 2^POWER
    static constexpr float FRACTION = 127.f / 128.f;
};
struct E4m3Code {
    static constexpr int POWER = 9;
    static constexpr float FRACTION = 0.875f;
};

typedef float float2c __attribute__((ext_vector_type(2)));

// four codes of a word as numbers (exact)
template <typename F>
__device__ __forceinline__ void decode4(unsigned w, float (&x)[4])
{
    if constexpr (std::is_same<F, Int8Code>::value) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (float)(int)(int8_t)(w >> (8 * i));
    } else {
        const float2c a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
    }
}

// four numbers, at most the format's largest in absolute value, as codes to nearest even
template <typename F>
__device__ __forceinline__ unsigned encode4(const float (&x)[4])
{
    if constexpr (std::is_same<F, Int8Code>::value) {
        unsigned w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w |= ((unsigned)(int)__builtin_rintf(x[i]) & 0xffu) << (8 * i);
        return w;
    } else {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
        return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
    }
}

// The exponent that a largest absolute value `top` needs: the smallest e >= EXP_LEAST with top <= FRACTION 2^POWER 2^e; EXP_NAN for a `top` that is
// not finite
template <typename F>
__device__ __forceinline__ int exponent_of(float top)
{
    if (!(top < INFINITY)) return EXP_NAN;
    const int x = __builtin_amdgcn_frexp_expf(top);       // top = f 2^x, f in [1/2, 1)
    const float f = __builtin_amdgcn_frexp_mantf(top);
    return top > 0.f ? max(x - F::POWER + (f > F::FRACTION ? 1 : 0), EXP_LEAST) : EXP_LEAST;
}

// of two exponents that rows need: the one that serves both
__device__ inline int exponent_join(int a, int b) { return a == EXP_NAN || b == EXP_NAN ? EXP_NAN : max(a, b); }

}  // namespace llla
