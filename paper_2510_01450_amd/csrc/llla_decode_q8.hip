// Decode over an 8-bit cache: one pass over the cache, the method of llla_mfma_decode.hip (moments relative to a reference exponent,
// records, merge and solve), with operands made of codes.
//
// A code times a power of two is an f16 number, so keys and values are operands of 16-bit matrix instructions as they are; only the
// weighted key x = w k is rounded.  Two variants, chosen per sequence:
//   two terms: x = h + l, l = x - h rounded (22 bits and the sign of l), weights in fp32.  The products of 32 keys start from zero and are then
//              added, one rounding of the sum for them: the precision of fp32 (which six products per tile give for fp32 rows).  For fp32 results,
//              and for sequences of at most 4 d keys, where only the ridge holds some directions and rounding x to 11 bits is not small against it.
//   one term:  w rounded to f16, and that same number used in every moment; x = w k rounded to f16.  2.5e-4 of the result, a seventh of the rounding of
//              a bf16 result.
// f16 has few exponents, so everything is relative: operands are k 2^-(E + U), E the largest exponent of the blocks that the wave reads and U the format's
// unit, which puts the largest code at 1/4; weights are relative to 2^R, R following the largest logit such that |w k| stays below 2^16.  The
// least number of f16, 2^-24, is then 2^-37 of the largest x and 2^-22 of the largest key.
//
// What bounds it: at d = 64 the cache's traffic and the vector work beside it (512 heads x 32768 int8 keys 415 us, 5.2 TB/s: vector port 56 % and matrix
// cores 34 % of the time, HBM at what a plain copy reaches; bf16 rows take 647).  At d = 128, four query heads to a cache head, the vector work: a
// wave converts nearly every block of keys and values for its 25 products (256 heads x 2048..16384 e4m3 keys 220 us with the merge; vector port 52 %,
// matrix cores 26 %, eight waves per compute unit).  Few heads: two launches, of which the merge is half (16 x 4096 23.4 us).
//
// Rows come by DMA into LDS, a block of 64 keys (one exponent) per stage, in 16-byte chunks whose order is permuted so that the transposed reads
// (ds_read_b64_tr_b8: eight keys of one feature per lane, which is an operand's order) have no bank conflicts.  int8: the low halves of 16-bit fields
// are f16 numbers u 2^-24 (subnormal, u = code + 128), which one packed multiply-add turns into (u - 128) 2^-9 r, r the block's power relative
// to E; e4m3 has a conversion with a scale.
#include "llla_cache.hpp"
#include "llla_decode_tail.hpp"

namespace llla {

// keys or values of one block for dual_row
template <typename F>
struct CodeRows {
    const uint8_t *p;
    float power;
};
template <typename F>
__device__ inline CodeRows<F> operator+(CodeRows<F> r, int64_t offset) { return CodeRows<F>{r.p + offset, r.power}; }
template <typename F>
__device__ inline float ld_f32(CodeRows<F> r, int c)
{
    if constexpr (std::is_same<F, Int8Code>::value) return r.power * (float)(int)(int8_t)r.p[c];
    else return r.power * __builtin_amdgcn_cvt_f32_fp8((int)r.p[c], 0);
}

namespace {

using namespace mfma;

constexpr int NT = DEC_NT, KEYS = CACHE_BLOCK;            // keys of a stage

template <int D>
struct Q8Shape : DecShape<D> {
    static constexpr bool TEAM = D == 128;                // four waves share one key stream
    static constexpr int NR = TEAM ? 2 : D / 16;          // row blocks of a wave
    static constexpr int NBUF = D <= 32 ? 4 : TEAM ? 1 : 2;
    static constexpr int KEYS_MIN = TEAM ? 256 : 512;     // fewest keys worth a workgroup
    static constexpr int SLOTS = D <= 32 ? 1024 : 512;    // workgroups worth having at once
    static constexpr int MAX_SPLIT = 32;
    static constexpr int CPR = D / 16;                    // 16-byte chunks of a row
    static constexpr int TILE_B = KEYS * D;               // keys or values of a stage
    static constexpr int DMAS = TILE_B / 1024;            // transfers of a tile
    static constexpr int STAGES = 2;
};

// value = operand * 2^(E + UNIT); weights of one term are f16 numbers, of two terms reach 2^17
template <typename F> struct Unit;
template <> struct Unit<Int8Code> { static constexpr int EXP = 9; };
template <> struct Unit<E4m3Code> { static constexpr int EXP = 11; };
constexpr int SLACK = 2;                                  // the reference moves when a logit exceeds what it was made for by more than this
template <bool TWO> constexpr int TOP = TWO ? 15 : 13;    // the largest weight when it moves

typedef _Float16 half2q __attribute__((ext_vector_type(2)));
typedef int int2q __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) int2q *lds_int2;

// eight codes (eight keys of a feature) as an operand; r, z: the block's power relative to E, for int8 as the factor and the addend of u 2^-24
struct BlockPower { float r; half2q s, z; };
template <typename F>
__device__ __forceinline__ BlockPower block_power(int below)
{
    BlockPower b;
    if constexpr (std::is_same<F, Int8Code>::value) {
        b.r = __builtin_ldexpf(1.f, -below);
        const _Float16 s = (_Float16)(b.r * 32768.f), z = (_Float16)(b.r * -0.25f);
        b.s = half2q{s, s};
        b.z = half2q{z, z};
    } else {
        b.r = __builtin_ldexpf(1.f, -11 - below);
        b.s = b.z = half2q{0, 0};
    }
    return b;
}
template <typename F>
__device__ __forceinline__ half8 operand(int2q c, const BlockPower &b)
{
    half8 o;
    if constexpr (std::is_same<F, Int8Code>::value) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const unsigned u = (unsigned)c[i] ^ 0x80808080u;
            const half2q lo = __builtin_elementwise_fma(__builtin_bit_cast(half2q, __builtin_amdgcn_perm(0u, u, 0x0c010c00u)), b.s, b.z);
            const half2q hi = __builtin_elementwise_fma(__builtin_bit_cast(half2q, __builtin_amdgcn_perm(0u, u, 0x0c030c02u)), b.s, b.z);
            o[4 * i] = lo[0]; o[4 * i + 1] = lo[1]; o[4 * i + 2] = hi[0]; o[4 * i + 3] = hi[1];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const half2q lo = __builtin_bit_cast(half2q, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((unsigned)c[i], b.r, false));
            const half2q hi = __builtin_bit_cast(half2q, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((unsigned)c[i], b.r, true));
            o[4 * i] = lo[0]; o[4 * i + 1] = lo[1]; o[4 * i + 2] = hi[0]; o[4 * i + 3] = hi[1];
        }
    }
    return o;
}

// sums of p[0..3] over the 16 lanes of a row; lane n receives the sum of p[n & 3]
__device__ __forceinline__ float reduce4(const float *p, int nn)
{
    const bool b0 = (nn & 1) != 0, b1 = (nn & 2) != 0;
    const float s0 = (b0 ? p[1] : p[0]) + dpp_f<0xB1>(b0 ? p[0] : p[1]);
    const float s1 = (b0 ? p[3] : p[2]) + dpp_f<0xB1>(b0 ? p[2] : p[3]);
    float s = (b1 ? s1 : s0) + dpp_f<0x4E>(b1 ? s0 : s1);
    s += dpp_f<0x124>(s);                                 // row_ror:4
    s += dpp_f<0x128>(s);                                 // row_ror:8
    return s;
}

// pairs of lanes 0 to 3 of the row
__device__ __forceinline__ half8 pair_bcast(half2q p)
{
    const float f = __builtin_bit_cast(float, p);
    const f32x4 v = {row_bcast<0>(f), row_bcast<1>(f), row_bcast<2>(f), row_bcast<3>(f)};
    return __builtin_bit_cast(half8, v);
}

// sum of a[0..7] b[0..7] onto c (v_dot2_f32_f16: exact products)
__device__ __forceinline__ float dot8(half8 a, half8 b, float c)
{
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        c = __builtin_amdgcn_fdot2(h2{a[i], a[i + 1]}, h2{b[i], b[i + 1]}, c, false);
    }
    return c;
}

// The value from here on is another one to the compiler: neither what was computed from it is kept for later, nor is a sum put off with its terms kept
__device__ __forceinline__ void pin(half8 &x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void pin(f32x4 &x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void pin(float &x) { asm volatile("" : "+v"(x)); }

// w k = h + l in two f16.  h is pinned between the two: the compiler (ROCm 7.2) otherwise forms some of its elements twice, for the operand from the
// product rounded to fp32 and for the remainder from the exact one (v_fma_mixlo), and where the two roundings differ, once in 2^14, h + l is off by 2^-11.
__device__ __forceinline__ void two_terms(const float (&w)[8], const half8 &k, half8 &h, half8 &l)
{
#pragma unroll
    for (int c = 0; c < 8; ++c) h[c] = (_Float16)(w[c] * (float)k[c]);
    pin(h);
#pragma unroll
    for (int c = 0; c < 8; ++c) l[c] = (_Float16)fmaf(w[c], (float)k[c], -(float)h[c]);
}

struct Q8Args {
    const char *K, *V;
    llla_strides sk, sv;
    const int8_t *ke, *ve;
    int HC, group, blocks;
    DecSplit split;
    HeadOut out;
    float cscale;
    float *parts;
};

template <int N>
__device__ __forceinline__ void wait_but() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// One wave's share of a piece, d <= 64
template <int D, typename F, typename TQ, bool FUSED, bool TWO, class Lds>
__device__ __forceinline__ void decode_q8_body(const Q8Args &a, const DecPiece &pc, Lds &lds, unsigned char *stages, int wave, int lane)
{
    using S = Q8Shape<D>;
    constexpr int NB = S::NB, U = Unit<F>::EXP, CPR = S::CPR, DMAS = S::DMAS;
    const int g = lane / 16, nn = lane % 16;
    const int L = pc.L, b = pc.b, bh = pc.bh, hc = pc.h / a.group;
    // shares begin at blocks of the format
    const int p0 = min((pc.k0 + KEYS - 1) & ~(KEYS - 1), L), p1 = pc.k1 >= L ? L : min((pc.k1 + KEYS - 1) & ~(KEYS - 1), L);
    const int share = ((p1 - p0 + 3) / 4 + KEYS - 1) / KEYS * KEYS;
    const int r0 = __builtin_amdgcn_readfirstlane(min(p0 + wave * share, p1));
    const int r1 = __builtin_amdgcn_readfirstlane(min(r0 + share, p1));
    const int nsteps = (r1 - r0 + KEYS - 1) / KEYS, b0 = r0 / KEYS;
    const char *Kh = a.K + b * a.sk.batch + hc * a.sk.head, *Vh = a.V + b * a.sv.batch + hc * a.sv.head;
    const int64_t krow = a.sk.seq, vrow = a.sv.seq;
    const int8_t *ke = a.ke + (size_t)(b * a.HC + hc) * a.blocks + b0, *ve = a.ve + (size_t)(b * a.HC + hc) * a.blocks + b0;

    // one term: mu~ and sum w v come from the matrix cores too, as products with a row block of weights (in every row of muw, yvw)
    f32x4 acc[S::NTILES], muw[NB], yvw[NB];
    float mu[NB], yv[NB], q[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) muw[i] = yvw[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < S::NTILES; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NB; ++i) { mu[i] = 0.f; yv[i] = 0.f; }
    float om = 0.f, mref = -INFINITY, mtrue = -INFINITY;
    int EK = EXP_NAN, EV = EXP_NAN;                       // largest exponents of the blocks read

    // Transfers: lane l brings chunk position l % CPR of key l / CPR of a group of 64 / CPR keys; the chunk of a row that lies at position p is
    // p ^ turn(key), turn the same for the same lane in every group.
    constexpr int KPD = 64 / CPR;
    const int dkey = lane / CPR, dchunk = (lane % CPR) ^ (D == 64 ? lane / 16 : D == 32 ? (lane / 16) & 1 : 0);
    unsigned char *const mine = stages + wave * (2 * S::STAGES * S::TILE_B);
    const unsigned mine_off = lds_offset(mine);
    const unsigned koff = (unsigned)(dkey * (int)krow + 16 * dchunk), voff = (unsigned)(dkey * (int)vrow + 16 * dchunk);
    // Waves that start together on equally spaced addresses would keep hitting the same memory channels in step: each begins at another block
    // of its share and wraps around.
    const int rot = nsteps > 0 ? __builtin_amdgcn_readfirstlane((int)(((unsigned)pc.rec * 4u + wave) * 7u % (unsigned)nsteps)) : 0;
    auto block_of = [&](int s) { const int t = s + rot; return t >= nsteps ? t - nsteps : t; };
    auto fetch = [&](int s, int stage, int tile) {        // tile: 0 keys, 1 values
        const int j0 = r0 + block_of(s) * KEYS;
        const unsigned dst = mine_off + (unsigned)((2 * stage + tile) * S::TILE_B);
        const char *X = tile ? Vh : Kh;
        const int64_t pitch = tile ? vrow : krow;
        if (j0 + KEYS <= L) {
            const char *p = X + j0 * pitch;
#pragma unroll
            for (int t = 0; t < DMAS; ++t) dma16_base_nt_off(p + t * KPD * pitch, tile ? voff : koff, dst + 1024u * t);
        } else {                                          // rows beyond the sequence: its last row (their weights are 0)
#pragma unroll
            for (int t = 0; t < DMAS; ++t) dma16_nt_off(X + min(j0 + t * KPD + dkey, L - 1) * pitch + 16 * dchunk, dst + 1024u * t);
        }
    };
    // transposed reads: lane (g, j) addresses eight bytes of one key and receives eight keys of feature 16 I + j: slot 2 e + c is key 8 g + 4 c + e, so
    // that a pair of slots is a pair of weights of one lane (below)
    const int tkey = 8 * g + 4 * ((nn / 2) & 1) + nn / 4, turn = D == 64 ? (tkey >> 2) & 3 : D == 32 ? (tkey >> 3) & 1 : 0;
    auto read = [&](int stage, int tile, int half, int I) {
        const unsigned at = (unsigned)(tkey * D + 16 * (I ^ turn) + 8 * (nn & 1));
        const unsigned char *p = mine + stage * 2 * S::TILE_B + tile * S::TILE_B + half * 32 * D;
        return __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_int2)(lds_void_ptr)(p + at));
    };

    if (nsteps > 0) {
        // in the order in which they are waited for
        fetch(0, 0, 0);
        fetch(0, 0, 1);
        if (nsteps > 1) { fetch(1, 1, 0); fetch(1, 1, 1); }
        {
            const TQ *qp = static_cast<const TQ *>(a.out.q) + (size_t)bh * D + nn;
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                if constexpr (sizeof(TQ) == 2) q[i] = bf16_to_f32(qp[16 * i]) * a.cscale;
                else q[i] = qp[16 * i] * a.cscale;
            }
        }
        for (int i = lane; i < nsteps; i += 64) {
            EK = max(EK, (int)ke[i]);
            EV = max(EV, (int)ve[i]);
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            EK = max(EK, __shfl_xor(EK, off));
            EV = max(EV, __shfl_xor(EV, off));
        }
        EK = __builtin_amdgcn_readfirstlane(EK);
        EV = __builtin_amdgcn_readfirstlane(EV);
#pragma unroll
        for (int i = 0; i < NB; ++i) q[i] = __builtin_ldexpf(q[i], EK + U);

        int ek64 = 0, ev64 = 0, have = -1;                // exponents of 64 blocks, one per lane; which 64
        auto compute = [&](int s, auto stage_tag) {
            constexpr int stage = decltype(stage_tag)::value;
            const int blk = block_of(s), j0 = r0 + blk * KEYS;
            if (blk / 64 != have) {
                have = blk / 64;
                const int i = min(64 * have + lane, nsteps - 1);
                ek64 = ke[i];
                ev64 = ve[i];
            }
            const int e_k = __builtin_amdgcn_readlane(ek64, blk % 64), e_v = __builtin_amdgcn_readlane(ev64, blk % 64);
            const BlockPower pk = block_power<F>(EK - e_k), pv = block_power<F>(EV - e_v);
            if (s + 1 < nsteps) wait_but<3 * DMAS>();     // all but this block's values and the next block
            else wait_but<DMAS>();
            half8 k[2][NB];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int I = 0; I < NB; ++I) k[h][I] = operand<F>(read(stage, 0, h, I), pk);
            if (s + 2 < nsteps) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // read before the transfer that overwrites them is requested
                fetch(s + 2, stage, 0);
            }
            float t[4];                                   // logit (log2 units) of key 32 h + 8 g + 4 c + (n % 4) in t[2 h + c]
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float p[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[e] = 0.f;
#pragma unroll
                        for (int I = 0; I < NB; ++I) p[e] = fmaf((float)k[h][I][2 * e + c], q[I], p[e]);
                    }
                    t[2 * h + c] = reduce4(p, nn);
                }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int I = 0; I < NB; ++I) pin(k[h][I]);
            if (e_k == EXP_NAN || e_v == EXP_NAN) t[0] = t[1] = t[2] = t[3] = NAN;      // (a scalar branch)
            if (j0 + KEYS > r1) {                         // (scalar branches)
#pragma unroll
                for (int i = 0; i < 4; ++i) t[i] = j0 + 32 * (i / 2) + 8 * g + 4 * (i % 2) + (nn & 3) < r1 ? t[i] : -INFINITY;
            }
            const float top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
            if (__builtin_amdgcn_ballot_w64(top > mref + (TOP<TWO> + SLACK)) != 0) {
                const float mnew = wave_max_dpp(top) - TOP<TWO>;
                const float alpha = mref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mref - mnew);
                mref = mnew;
                om *= alpha;
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    if constexpr (TWO) { mu[i] *= alpha; yv[i] *= alpha; }
                    else { muw[i] *= alpha; yvw[i] *= alpha; }
                }
#pragma unroll
                for (int i = 0; i < S::NTILES; ++i) acc[i] *= alpha;
            }
            mtrue = fmaxf(mtrue, top);
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = __builtin_amdgcn_exp2f(t[i] - mref);           // exp2(-inf) = 0 masks the tail
                if constexpr (!TWO) w[i] = (float)(_Float16)w[i];
                om += w[i];
            }
            if (s + 2 < nsteps) wait_but<3 * DMAS>();     // all but the next block and the keys of the one after it
            else if (s + 1 < nsteps) wait_but<2 * DMAS>();
            else wait_but<0>();
            // (the scheduler is kept inside one block of features: left to itself it reads and converts the whole stage first and spills)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                int2q raw[NB];                            // values, on their way while the keys are multiplied
#pragma unroll
                for (int J = 0; J < NB; ++J) raw[J] = read(stage, 1, h, J);
                half8 w8, x[NB], xl[NB];                  // the half's weights in the operands' order: w8 with one term, wc (and xl) with two
                float wc[8];
                if constexpr (!TWO) w8 = pair_bcast(half2q{(_Float16)w[2 * h], (_Float16)w[2 * h + 1]});
                else {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        wc[c] = row_bcast<0>(w[2 * h + c]);
                        wc[2 + c] = row_bcast<1>(w[2 * h + c]);
                        wc[4 + c] = row_bcast<2>(w[2 * h + c]);
                        wc[6 + c] = row_bcast<3>(w[2 * h + c]);
                    }
                }
                auto product = [&](int I, const half8 &b, f32x4 &sum) {
                    if constexpr (!TWO) sum = mfma_f16(x[I], b, sum);
                    else {
                        sum += mfma_f16(x[I], b, mfma_f16(xl[I], b, f32x4{0.f, 0.f, 0.f, 0.f}));
                        pin(sum);
                    }
                };
#pragma unroll
                for (int J = 0; J < NB; ++J) {
                    if constexpr (!TWO) {
                        x[J] = w8 * k[h][J];
                        muw[J] = mfma_f16(w8, k[h][J], muw[J]);
                    } else {
                        two_terms(wc, k[h][J], x[J], xl[J]);
#pragma unroll
                        for (int c = 0; c < 8; ++c) mu[J] = fmaf(wc[c], (float)k[h][J][c], mu[J]);
                    }
#pragma unroll
                    for (int I = 0; I <= J; ++I) product(I, k[h][J], acc[upper_tile<NB>(I, J)]);
                    if constexpr (TWO) pin(mu[J]);
                    pin(x[J]);
                    if constexpr (TWO) pin(xl[J]);
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int J = 0; J < NB; ++J) {
                    const half8 v = operand<F>(raw[J], pv);
                    if constexpr (!TWO) yvw[J] = mfma_f16(w8, v, yvw[J]);
                    else {
#pragma unroll
                        for (int c = 0; c < 8; ++c) yv[J] = fmaf(wc[c], (float)v[c], yv[J]);
                    }
#pragma unroll
                    for (int I = 0; I < NB; ++I) product(I, v, acc[S::NSIG + NB * I + J]);
                    if constexpr (TWO) pin(yv[J]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (s + 2 < nsteps) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                fetch(s + 2, stage, 1);
            }
        };
#pragma unroll 1
        for (int s = 0; s < nsteps; s += 2) {
            compute(s, std::integral_constant<int, 0>{});
            if (s + 1 < nsteps) compute(s + 1, std::integral_constant<int, 1>{});
        }
        if constexpr (!TWO) {
#pragma unroll
            for (int i = 0; i < NB; ++i) { mu[i] = 0.25f * muw[i][0]; yv[i] = 0.25f * yvw[i][0]; }      // (summed over the four groups below)
        }
        // back from the operands' scale
#pragma unroll
        for (int t = 0; t < S::NTILES; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][i] = __builtin_ldexpf(acc[t][i], EK + U + (t < S::NSIG ? EK : EV) + U);
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            mu[i] = __builtin_ldexpf(mu[i], EK + U);
            yv[i] = __builtin_ldexpf(yv[i], EV + U);
        }
    }

    __syncthreads();                                      // the stages of all waves are dead: the merge takes their place
    mtrue = wave_max_dpp(mtrue);
    om += dpp_f<0xB1>(om);
    om += dpp_f<0x4E>(om);
    om = rows_allsum(om);
#pragma unroll
    for (int i = 0; i < NB; ++i) { mu[i] = rows_allsum(mu[i]); yv[i] = rows_allsum(yv[i]); }
    float *R = a.parts + (size_t)pc.rec * S::REC_F;       // this workgroup's record (not FUSED)
    finish_workgroup<D, TQ, false, FUSED, S::NBUF>(lds, acc, mu, yv, om, mref, mtrue, R, a.out, bh, wave, lane);
}

// d = 128: the four waves of a workgroup share a key stream.  Wave W owns row blocks W and 7 - W of the moments (25 tiles whatever W) and forms of the
// keys and values what it multiplies with; logits it sums over its own two feature blocks, one stage ahead, and the four partial sums meet in LDS.  One
// barrier per stage: behind it the next stage's rows are there, this stage's partial logits are, and the stage before last is free for a transfer.
constexpr int WIDE_STAGES = 4, WIDE_STAGE_B = 2 * KEYS * 128;
struct WideLds {
    unsigned char rows[WIDE_STAGES][WIDE_STAGE_B];
    float part[2][KEYS][4];
};

template <typename F, typename TQ, bool FUSED, bool TWO, int W, class Lds>
__device__ __forceinline__ void decode_q8_wide_body(const Q8Args &a, const DecPiece &pc, Lds &lds, WideLds &wl, int wave, int lane)
{
    constexpr int D = 128, NB = 8, NR = 2, U = Unit<F>::EXP;
    using S = Q8Shape<D>;
    constexpr int row[NR] = {W, 7 - W}, low = W < 4 ? W : 7 - W;
    const int g = lane / 16, nn = lane % 16;
    const int L = pc.L, b = pc.b, bh = pc.bh, hc = pc.h / a.group;
    const int r0 = __builtin_amdgcn_readfirstlane(min((pc.k0 + KEYS - 1) & ~(KEYS - 1), L));
    const int r1 = __builtin_amdgcn_readfirstlane(pc.k1 >= L ? L : min((pc.k1 + KEYS - 1) & ~(KEYS - 1), L));
    const int nsteps = (r1 - r0 + KEYS - 1) / KEYS, b0 = r0 / KEYS;
    const char *Kh = a.K + b * a.sk.batch + hc * a.sk.head, *Vh = a.V + b * a.sv.batch + hc * a.sv.head;
    const int64_t krow = a.sk.seq, vrow = a.sv.seq;
    const int8_t *ke = a.ke + (size_t)(b * a.HC + hc) * a.blocks + b0, *ve = a.ve + (size_t)(b * a.HC + hc) * a.blocks + b0;

    f32x4 acc[S::NTILES];                                 // the tiles of row blocks row[0] and row[1] only
    float mu[NR], yv[NR], q[NR];
#pragma unroll
    for (int t = 0; t < S::NTILES; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NR; ++i) { mu[i] = 0.f; yv[i] = 0.f; }
    auto for_tiles = [&](auto fn) {
#pragma unroll
        for (int i = 0; i < NR; ++i) {
#pragma unroll
            for (int J = row[i]; J < NB; ++J) fn(upper_tile<NB>(row[i], J), true);
#pragma unroll
            for (int J = 0; J < NB; ++J) fn(S::NSIG + NB * row[i] + J, false);
        }
    };
    float om = 0.f, mref = -INFINITY, mtrue = -INFINITY;
    int EK = EXP_NAN, EV = EXP_NAN;

    // transfers: of the eight of a tile (eight keys each) wave W brings numbers 2 W and 2 W + 1
    const int dkey = lane / 8, dchunk = (lane % 8) ^ (lane / 16);
    const unsigned koff = (unsigned)(dkey * (int)krow + 16 * dchunk), voff = (unsigned)(dkey * (int)vrow + 16 * dchunk);
    const unsigned rows_off = lds_offset(wl.rows);
    const int rot = nsteps > 0 ? __builtin_amdgcn_readfirstlane((int)((unsigned)pc.rec * 7u % (unsigned)nsteps)) : 0;
    auto block_of = [&](int s) { const int t = s + rot; return t >= nsteps ? t - nsteps : t; };
    auto fetch = [&](int s) {
        const int j0 = r0 + block_of(s) * KEYS;
        const unsigned dst = rows_off + (unsigned)((s & (WIDE_STAGES - 1)) * WIDE_STAGE_B);
#pragma unroll
        for (int tile = 0; tile < 2; ++tile) {
            const char *X = tile ? Vh : Kh;
            const int64_t pitch = tile ? vrow : krow;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int t = 2 * W + i;
                const unsigned to = dst + (unsigned)(tile * KEYS * D + 1024 * t), turn = 64u * i;      // (odd groups: the other half of the chunks)
                if (j0 + KEYS <= L) dma16_base_nt_off(X + (j0 + 8 * t) * pitch, (tile ? voff : koff) ^ turn, to);
                else dma16_nt_off(X + min(j0 + 8 * t + dkey, L - 1) * pitch + (16 * dchunk ^ turn), to);
            }
        }
    };
    const int tkey = 8 * g + nn / 2, turn = 4 * (g & 1) + (nn >> 2);
    auto read = [&](int s, int tile, int half, int I) {
        const unsigned at = (unsigned)((32 * half + tkey) * D + 16 * (I ^ turn) + 8 * (nn & 1));
        return __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_int2)(lds_void_ptr)(wl.rows[s & (WIDE_STAGES - 1)] + tile * KEYS * D + at));
    };

    if (nsteps > 0) {
        fetch(0);
        if (nsteps > 1) fetch(1);
        if (nsteps > 2) fetch(2);
        {
            const TQ *qp = static_cast<const TQ *>(a.out.q) + (size_t)bh * D + nn;
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                if constexpr (sizeof(TQ) == 2) q[i] = bf16_to_f32(qp[16 * row[i]]) * a.cscale;
                else q[i] = qp[16 * row[i]] * a.cscale;
            }
        }
        for (int i = lane; i < nsteps; i += 64) {
            EK = max(EK, (int)ke[i]);
            EV = max(EV, (int)ve[i]);
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            EK = max(EK, __shfl_xor(EK, off));
            EV = max(EV, __shfl_xor(EV, off));
        }
        EK = __builtin_amdgcn_readfirstlane(EK);
        EV = __builtin_amdgcn_readfirstlane(EV);
#pragma unroll
        for (int i = 0; i < NR; ++i) q[i] = __builtin_ldexpf(q[i], EK + U);

        int ek64 = 0, ev64 = 0, have = -1;
        BlockPower pk, pv;
        bool marked = false;
        half8 kown[2][NR];
        auto partial_logits = [&](int s) {                // and the operands of this wave's row blocks
            const int blk = block_of(s);
            if (blk / 64 != have) {
                have = blk / 64;
                const int i = min(64 * have + lane, nsteps - 1);
                ek64 = ke[i];
                ev64 = ve[i];
            }
            const int e_k = __builtin_amdgcn_readlane(ek64, blk % 64), e_v = __builtin_amdgcn_readlane(ev64, blk % 64);
            pk = block_power<F>(EK - e_k);
            pv = block_power<F>(EV - e_v);
            marked = e_k == EXP_NAN || e_v == EXP_NAN;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int i = 0; i < NR; ++i) kown[h][i] = operand<F>(read(s, 0, h, row[i]), pk);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float p[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[e] = fmaf((float)kown[h][1][4 * c + e], q[1], (float)kown[h][0][4 * c + e] * q[0]);
                    const float t = reduce4(p, nn);
                    if (c == 1) { pin(kown[h][0]); pin(kown[h][1]); }
                    if (nn < 4) wl.part[s & 1][32 * h + 8 * g + 4 * c + nn][W] = t;
                }
            }
        };
        auto meet = [&](bool later) {                     // later: the next stage but one is still on its way
            if (later) wait_but<4>();
            else wait_but<0>();
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        };
        if (nsteps > 2) wait_but<8>();
        else if (nsteps > 1) wait_but<4>();
        else wait_but<0>();
        asm volatile("s_barrier" ::: "memory");
        partial_logits(0);
#pragma unroll 1
        for (int s = 0; s < nsteps; ++s) {
            meet(s + 2 < nsteps);
            if (s + 3 < nsteps) fetch(s + 3);
            const int j0 = r0 + block_of(s) * KEYS;
            // a half's codes, requested long before they are multiplied: the first half's here, the second's when the first's keys are done
            int2q kraw[NB], vraw[NB];
            auto request = [&](int h) {
#pragma unroll
                for (int J = low; J < NB; ++J)
                    if (J != row[0] && J != row[1]) kraw[J] = read(s, 0, h, J);
#pragma unroll
                for (int J = 0; J < NB; ++J) vraw[J] = read(s, 1, h, J);
            };
            request(0);
            float t[4];                                   // logit of key 32 h + 8 g + 2 (n % 4) + c in t[2 h + c]: a lane's pair is a pair of an operand
            const int key = 8 * g + 2 * (nn & 3);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 p = *reinterpret_cast<const f32x4 *>(wl.part[s & 1][32 * (i / 2) + key + i % 2]);
                t[i] = (p[0] + p[1]) + (p[2] + p[3]);
            }
            if (marked) t[0] = t[1] = t[2] = t[3] = NAN;  // (scalar branches)
            if (j0 + KEYS > r1) {
#pragma unroll
                for (int i = 0; i < 4; ++i) t[i] = j0 + 32 * (i / 2) + key + i % 2 < r1 ? t[i] : -INFINITY;
            }
            const float top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
            if (__builtin_amdgcn_ballot_w64(top > mref + (TOP<TWO> + SLACK)) != 0) {
                const float mnew = wave_max_dpp(top) - TOP<TWO>;
                const float alpha = mref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mref - mnew);
                mref = mnew;
                om *= alpha;
#pragma unroll
                for (int i = 0; i < NR; ++i) { mu[i] *= alpha; yv[i] *= alpha; }
                for_tiles([&](int i, bool) { acc[i] *= alpha; });
            }
            mtrue = fmaxf(mtrue, top);
            float w[4];
            half2q wp[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_exp2f(t[i] - mref);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (TWO) om += w[2 * h] + w[2 * h + 1];
                else {
                    wp[h] = half2q{(_Float16)w[2 * h], (_Float16)w[2 * h + 1]};
                    om = __builtin_amdgcn_fdot2(wp[h], half2q{(_Float16)1.f, (_Float16)1.f}, om, false);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                half8 x[NR], xl[NR], w8;                  // the half's weights in the operands' order: w8 with one term, wc (and xl) with two
                float wc[8];
                if constexpr (!TWO) w8 = pair_bcast(wp[h]);
                else {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        wc[c] = row_bcast<0>(w[2 * h + c]);
                        wc[2 + c] = row_bcast<1>(w[2 * h + c]);
                        wc[4 + c] = row_bcast<2>(w[2 * h + c]);
                        wc[6 + c] = row_bcast<3>(w[2 * h + c]);
                    }
                }
#pragma unroll
                for (int i = 0; i < NR; ++i) {
                    if constexpr (!TWO) {
                        x[i] = w8 * kown[h][i];
                        mu[i] = dot8(w8, kown[h][i], mu[i]);
                    } else {
                        two_terms(wc, kown[h][i], x[i], xl[i]);
#pragma unroll
                        for (int c = 0; c < 8; ++c) mu[i] = fmaf(wc[c], (float)kown[h][i][c], mu[i]);
                    }
                }
                auto product = [&](int i, const half8 &b, f32x4 &sum) {
                    if constexpr (!TWO) sum = mfma_f16(x[i], b, sum);
                    else {
                        sum += mfma_f16(x[i], b, mfma_f16(xl[i], b, f32x4{0.f, 0.f, 0.f, 0.f}));
                        pin(sum);
                    }
                };
#pragma unroll
                for (int i = 0; i < NR; ++i) {
                    pin(mu[i]);
                    pin(x[i]);
                    if constexpr (TWO) pin(xl[i]);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int J = low; J < NB; ++J) {
                    const half8 b = J == row[0] ? kown[h][0] : J == row[1] ? kown[h][1] : operand<F>(kraw[J], pk);
#pragma unroll
                    for (int i = 0; i < NR; ++i)
                        if (J >= row[i]) product(i, b, acc[upper_tile<NB>(row[i], J)]);
                    if (J % 2) __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int J = 0; J < NB; ++J) {
                    const half8 v = operand<F>(vraw[J], pv);
#pragma unroll
                    for (int i = 0; i < NR; ++i) {
                        if (J == row[i]) {
                            if constexpr (!TWO) yv[i] = dot8(w8, v, yv[i]);
                            else {
#pragma unroll
                                for (int c = 0; c < 8; ++c) yv[i] = fmaf(wc[c], (float)v[c], yv[i]);
                            }
                        }
                        product(i, v, acc[S::NSIG + NB * row[i] + J]);
                    }
                    if (J == row[0]) pin(yv[0]);
                    if (J == row[1]) pin(yv[1]);
                    if (J % 2) __builtin_amdgcn_sched_barrier(0);
                }
                if (h == 0) request(1);
            }
            if (s + 1 < nsteps) partial_logits(s + 1);
        }
        for_tiles([&](int t, bool sigma) {
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][i] = __builtin_ldexpf(acc[t][i], EK + U + (sigma ? EK : EV) + U);
        });
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            mu[i] = __builtin_ldexpf(mu[i], EK + U);
            yv[i] = __builtin_ldexpf(yv[i], EV + U);
        }
    }

    mtrue = wave_max_dpp(mtrue);
    om += dpp_f<0xB1>(om);
    om += dpp_f<0x4E>(om);
    om = rows_allsum(om);
#pragma unroll
    for (int i = 0; i < NR; ++i) { mu[i] = rows_allsum(mu[i]); yv[i] = rows_allsum(yv[i]); }
    if constexpr (FUSED) __syncthreads();                 // the rows are dead: the moments take their place
    // every wave's own tiles, relative to the true maximum
    const float f = mref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mref - mtrue);
    float *R = a.parts + (size_t)pc.rec * S::REC_F, *tiles, *mud, *yvd;
    if constexpr (FUSED) { tiles = lds.tiles[0]; mud = lds.mu[0]; yvd = lds.yv[0]; }
    else { tiles = R + S::HDR; mud = R + 64; yvd = R + 64 + D; }
    for_tiles([&](int t, bool) { *reinterpret_cast<f32x4 *>(tiles + t * 256 + lane * 4) = f * acc[t]; });
    if (g == 0) {
#pragma unroll
        for (int i = 0; i < NR; ++i) { mud[16 * row[i] + nn] = f * mu[i]; yvd[16 * row[i] + nn] = f * yv[i]; }
    }
    if (W == 0 && lane == 0) {
        if constexpr (FUSED) lds.om[0] = f * om;
        else { R[0] = mtrue; R[1] = f * om; }
    }
    if constexpr (FUSED) {
        const QueryPart<D> query = load_query<D, TQ, false>(a.out, bh, lane);
        __syncthreads();
        solve_head<D, TQ, false>(lds, a.out, query, bh, wave, lane);
    }
}

// LDS of a workgroup: the stages of its waves, later the moments
template <int D, bool FUSED>
struct Q8Lds {
    using S = Q8Shape<D>;
    using Head = HeadLds<D, S::NBUF, S::TEAM ? 1 : 4>;
    static constexpr size_t STAGES_B = S::TEAM ? sizeof(WideLds) : (size_t)4 * S::STAGES * 2 * S::TILE_B;
    static constexpr size_t BYTES = (FUSED || !S::TEAM) && sizeof(Head) > STAGES_B ? sizeof(Head) : STAGES_B;
};

template <int D, typename F, typename TQ, bool FUSED, bool TWO>
__device__ __forceinline__ void decode_q8_piece(const Q8Args &a, const DecPiece &pc, unsigned char *raw, int wave)
{
    auto &lds = *reinterpret_cast<typename Q8Lds<D, FUSED>::Head *>(raw);
    if constexpr (D == 128) {                             // scalar branches; all four waves meet at the same barriers
        WideLds &wl = *reinterpret_cast<WideLds *>(raw);
        if (wave == 0) decode_q8_wide_body<F, TQ, FUSED, TWO, 0>(a, pc, lds, wl, wave, piece_lane());
        else if (wave == 1) decode_q8_wide_body<F, TQ, FUSED, TWO, 1>(a, pc, lds, wl, wave, piece_lane());
        else if (wave == 2) decode_q8_wide_body<F, TQ, FUSED, TWO, 2>(a, pc, lds, wl, wave, piece_lane());
        else decode_q8_wide_body<F, TQ, FUSED, TWO, 3>(a, pc, lds, wl, wave, piece_lane());
    } else {
        decode_q8_body<D, F, TQ, FUSED, TWO>(a, pc, lds, raw, wave, piece_lane());
    }
}

// One term: sequences of at most PRECISE_KEYS are left to precise_heads_kernel (one kernel for both has not the registers).
template <int D> constexpr int PRECISE_KEYS = 4 * D;
template <int D, typename F, typename TQ, bool FUSED, bool TWO>
__global__ __launch_bounds__(NT, (D == 128 && FUSED) ? 1 : 2) void decode_q8_kernel(Q8Args a)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    __shared__ __align__(16) unsigned char raw[Q8Lds<D, FUSED>::BYTES];
    for_pieces<FUSED>(a.split, [&](const DecPiece &pc) {
        if (TWO || pc.L > PRECISE_KEYS<D>) decode_q8_piece<D, F, TQ, FUSED, TWO>(a, pc, raw, wave);
    });
}

// Sequences of at most 64 keys, which one block of the format holds: in key space (llla_dual.hpp); empty ones give zeros
template <int D, typename F, typename TQ, typename TO>
__device__ __forceinline__ void short_head(dual::DualShared<D, DUAL_MAX_KEYS> &sm, const Q8Args &a, float scale, int bh)
{
    const int H = a.split.H, b = bh / H, hc = bh % H / a.group, m = cache_length(a.split.seqlens, b, a.split.L_max);
    if (m > DUAL_MAX_KEYS) return;                        // the whole workgroup
    TO *o = static_cast<TO *>(a.out.o) + (size_t)bh * D;
    if (m == 0) {
        if (threadIdx.x < D) dual::st_out(o + threadIdx.x, 0.0);
        return;
    }
    const size_t at = (size_t)(b * a.HC + hc) * a.blocks;
    const int ek = a.ke[at], ev = a.ve[at];
    const CodeRows<F> K{reinterpret_cast<const uint8_t *>(a.K + b * a.sk.batch + hc * a.sk.head), ek == EXP_NAN ? NAN : __builtin_ldexpf(1.f, ek)};
    const CodeRows<F> V{reinterpret_cast<const uint8_t *>(a.V + b * a.sv.batch + hc * a.sv.head), ev == EXP_NAN ? NAN : __builtin_ldexpf(1.f, ev)};
    dual::dual_row<D, TQ, TO>(sm, static_cast<const TQ *>(a.out.q) + (size_t)bh * D, K, V, a.sk.seq, a.sv.seq, m, (double)a.out.lambda, scale, o,
                              nullptr, nullptr);
}

// Sequences that the kernels proper leave: one workgroup per head.  precise: also those that one term is too little for.
template <int D, typename F, typename TQ>
__global__ __launch_bounds__(NT) void precise_heads_kernel(Q8Args a, float scale, int precise)
{
    using Dual = dual::DualShared<D, DUAL_MAX_KEYS>;
    __shared__ __align__(16) unsigned char raw[Q8Lds<D, true>::BYTES > sizeof(Dual) ? Q8Lds<D, true>::BYTES : sizeof(Dual)];
    const int bh = blockIdx.x, H = a.split.H, L = __builtin_amdgcn_readfirstlane(cache_length(a.split.seqlens, bh / H, a.split.L_max));
    if (L <= DUAL_MAX_KEYS) {
        if (a.out.out_bf16) short_head<D, F, TQ, bf16_t>(*reinterpret_cast<Dual *>(raw), a, scale, bh);
        else short_head<D, F, TQ, float>(*reinterpret_cast<Dual *>(raw), a, scale, bh);
    } else if (precise && L <= PRECISE_KEYS<D>) {
        const DecPiece pc{bh / H, bh % H, bh, L, 0, L, bh};
        decode_q8_piece<D, F, TQ, true, true>(a, pc, raw, __builtin_amdgcn_readfirstlane(threadIdx.x / 64));
    }
}

// Merge of the records, one workgroup per head; least: shorter sequences are not of this call's
template <int D, typename TQ>
__global__ __launch_bounds__(NT, D == 128 ? 1 : 2) void merge_q8_kernel(DecSplit split, HeadOut out, const float *__restrict__ parts, int least)
{
    __shared__ HeadLds<D, 1, 1> lds;
    if (seq_len(split, blockIdx.x / split.H) <= least) return;
    merge_head<D, TQ, false>(lds, split, out, parts, blockIdx.x);
}

// ---- host -----------------------------------------------------------------------------------------------------------------------------
constexpr size_t MAX_RECORD_BYTES = (size_t)1 << 30;

// Workgroups per head of the even cut: rounds of the GPU's slots times the keys of a workgroup, and what a record costs
template <int D>
int q8_nsplit(int bh, int L)
{
    using S = Q8Shape<D>;
    int best = 1;
    double best_cost = 1e300;
    for (int ns = 1; ns <= S::MAX_SPLIT; ++ns) {
        if (ns > 1 && ((L + ns - 1) / ns < S::KEYS_MIN || (size_t)bh * ns * S::REC_F * sizeof(float) > MAX_RECORD_BYTES)) break;
        const double rounds = (double)(((long long)bh * ns + S::SLOTS - 1) / S::SLOTS);
        const double cost = rounds * ((double)L / ns + S::KEYS_MIN / 4) + (ns > 1 ? S::KEYS_MIN / 8 * ns : 0);
        if (cost < best_cost) { best_cost = cost; best = ns; }
    }
    return best;
}

template <int D>
size_t q8_records(int B, int H, int L)
{
    using S = Q8Shape<D>;
    const int ns = q8_nsplit<D>(B * H, L);
    size_t n = ns > 1 ? (size_t)B * H * ns : 0;
    const size_t flat = flat_records(B, H, S::SLOTS);
    if (B >= 2 && L > S::KEYS_MIN && flat * S::REC_F * sizeof(float) <= MAX_RECORD_BYTES) n = std::max(n, flat);
    return n;
}

template <int D>
size_t q8_bytes(int B, int H, int L) { return L <= DUAL_MAX_KEYS ? 0 : round_up(q8_records<D>(B, H, L) * Q8Shape<D>::REC_F * sizeof(float), 256); }

template <int D, typename F, typename TQ>
hipError_t q8_launch(const DecodeQ8Problem &p)
{
    using S = Q8Shape<D>;
    const llla_cache &c = p.c;
    const int bh = c.B * p.H;
    Q8Args a;
    a.K = static_cast<const char *>(c.K); a.V = static_cast<const char *>(c.V);
    a.sk = c.sk; a.sv = c.sv;
    a.ke = c.k_exp; a.ve = c.v_exp;
    a.HC = c.H; a.group = p.H / c.H; a.blocks = cache_blocks(c.L_max);
    a.out = HeadOut{p.q, p.o, p.out == LLLA_BF16 ? 1 : 0, p.lambda};
    a.cscale = p.scale * LOG2E;
    a.parts = static_cast<float *>(p.ws);
    Problem cut{};
    cut.seqlens = p.seqlens; cut.B = c.B; cut.H = p.H; cut.n = c.L_max;
    // which sequences are whose: at most DUAL_MAX_KEYS in key space; a bf16 result's others at most PRECISE_KEYS with two terms
    const bool two = p.out != LLLA_BF16 || c.L_max <= PRECISE_KEYS<D>;
    const int least = two ? DUAL_MAX_KEYS : PRECISE_KEYS<D>;
    if (c.L_max <= DUAL_MAX_KEYS) {
        a.split = DecSplit{p.seqlens, c.B, p.H, c.L_max, 1, 0, 0, 0, 0};
        stage_mark(p.stream, "decode_q8_short");
        hipLaunchKernelGGL((precise_heads_kernel<D, F, TQ>), dim3(bh), dim3(NT), 0, p.stream, a, p.scale, 0);
        return hipGetLastError();
    }
    const size_t records = q8_records<D>(c.B, p.H, c.L_max);
    const bool scratch = p.ws != nullptr && (reinterpret_cast<uintptr_t>(p.ws) & 255u) == 0 && p.ws_bytes >= records * S::REC_F * sizeof(float);
    const int ns = scratch ? q8_nsplit<D>(bh, c.L_max) : 1;
    a.split = choose_split(cut, ns, scratch ? records : 0, S::SLOTS, 2 * CACHE_BLOCK, S::KEYS_MIN, S::MAX_SPLIT);
    const bool fused = a.split.nsplit == 1 && a.split.slots == 0;
    const dim3 grid = fused ? dim3(1, bh) : a.split.slots ? dim3(a.split.slots, p.H) : dim3(a.split.nsplit, bh);
    stage_mark(p.stream, fused ? "decode_q8" : "decode_q8_partial");
    if (fused && two) hipLaunchKernelGGL((decode_q8_kernel<D, F, TQ, true, true>), grid, dim3(NT), 0, p.stream, a);
    else if (fused) hipLaunchKernelGGL((decode_q8_kernel<D, F, TQ, true, false>), grid, dim3(NT), 0, p.stream, a);
    else if (two) hipLaunchKernelGGL((decode_q8_kernel<D, F, TQ, false, true>), grid, dim3(NT), 0, p.stream, a);
    else hipLaunchKernelGGL((decode_q8_kernel<D, F, TQ, false, false>), grid, dim3(NT), 0, p.stream, a);
    if (!fused) {
        stage_mark(p.stream, "decode_q8_merge");
        hipLaunchKernelGGL((merge_q8_kernel<D, TQ>), dim3(bh), dim3(NT), 0, p.stream, a.split, a.out, (const float *)a.parts, p.seqlens ? least : 0);
    }
    // (behind the others: a fused kernel with two terms has written something for short sequences too)
    if (p.seqlens != nullptr)
        hipLaunchKernelGGL((precise_heads_kernel<D, F, TQ>), dim3(bh), dim3(NT), 0, p.stream, a, p.scale, two ? 0 : 1);
    return hipGetLastError();
}

template <int D>
hipError_t q8_by_type(const DecodeQ8Problem &p)
{
    if (p.c.type == LLLA_I8) return p.in == LLLA_F32 ? q8_launch<D, Int8Code, float>(p) : q8_launch<D, Int8Code, bf16_t>(p);
    return p.in == LLLA_F32 ? q8_launch<D, E4m3Code, float>(p) : q8_launch<D, E4m3Code, bf16_t>(p);
}

}  // namespace

size_t decode_q8_workspace_bytes(int B, int H, int L_max, int d)
{
    switch (d) {
        case 16: return q8_bytes<16>(B, H, L_max);
        case 32: return q8_bytes<32>(B, H, L_max);
        case 64: return q8_bytes<64>(B, H, L_max);
        case 128: return q8_bytes<128>(B, H, L_max);
        default: return 0;
    }
}

hipError_t decode_q8(const DecodeQ8Problem &p)
{
    switch (p.c.d) {
        case 16: return q8_by_type<16>(p);
        case 32: return q8_by_type<32>(p);
        case 64: return q8_by_type<64>(p);
        case 128: return q8_by_type<128>(p);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace llla
