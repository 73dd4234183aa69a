// Decode over an 8-bit cache: one pass over the cache, the method of llla_mfma_decode_f32.hip (its layout of rows in lanes, reference exponent,
// records, merge and solve), with operands made for codes.
//
// A code times a power of two is an f16 number, so keys and values are operands of 16-bit matrix instructions as they are; only the
// weighted key x = w k needs more bits and is taken in two f16 terms, x = h + l with l = x - h rounded (22 bits and the sign of l).  The second
// moment sum w k k^T and sum w k v^T then cost two products per tile, against six for fp32 rows, and carry the precision of fp32.
// f16 has few exponents, so everything is relative:  k16 = k 2^-(E + U), E the largest exponent of the blocks that the wave reads and U
// the format's unit (int8 codes land in +-1/4, e4m3 ones in +-57344); weights are relative to 2^R, R following the largest logit such that
// |w k16| stays below 2^16.  The least number of f16, 2^-24, is then 2^-38 of the largest x, and a block's codes are exact as long as its
// exponent is at most 15 (int8) or 22 (e4m3) below E.
//
// Lane (g, n) owns features NB n .. NB n + NB - 1 (NB = d / 16) of key g of a chunk of four: NB bytes.  Two chunks' words give the pairs of an
// operand: int8 bytes of both, each in the low half of a 16-bit field, are f16 numbers u 2^-24 (subnormal, u = code + 128), which one
// packed multiply-add turns into (u - 128) 2^-9 r, r the block's power relative to E; e4m3 has a conversion with a scale.
//
// A step is 32 keys of one block.  At d = 128 the four waves of a workgroup share a key stream and the row blocks of the moments (W and 7 - W
// each), and every wave forms the operands for itself.
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

constexpr int NT = DEC_NT, STEP = 32, CH = 8;

template <int D>
struct Q8Shape : DecShape<D> {
    static constexpr bool TEAM = D == 128;
    static constexpr int NR = TEAM ? 2 : D / 16;          // row blocks of a wave
    static constexpr int NBUF = D <= 32 ? 4 : TEAM ? 1 : 2;
    static constexpr int WORDS = D == 128 ? 2 : 1;        // words of a row that a lane owns
    static constexpr int KEYS_MIN = TEAM ? 256 : 512;     // fewest keys worth a workgroup
    static constexpr int SLOTS = 512;                     // workgroups worth having at once
    static constexpr int MAX_SPLIT = 32;
};

// value = operand * 2^(E + UNIT); weights reach 2^(TOP + 2), an operand times a weight 2^16
template <typename F> struct Unit;
template <> struct Unit<Int8Code> { static constexpr int EXP = 9, TOP = 15; };
template <> struct Unit<E4m3Code> { static constexpr int EXP = -7, TOP = -2; };

typedef _Float16 half2q __attribute__((ext_vector_type(2)));

template <int WORDS> struct Codes { unsigned u[WORDS]; };

template <int NB>
__device__ __forceinline__ Codes<(NB > 4 ? 2 : 1)> load_codes(const char *p)
{
    Codes<(NB > 4 ? 2 : 1)> c;
    if constexpr (NB == 1) c.u[0] = *reinterpret_cast<const uint8_t *>(p);
    else if constexpr (NB == 2) c.u[0] = *reinterpret_cast<const uint16_t *>(p);
    else if constexpr (NB == 4) c.u[0] = __builtin_nontemporal_load(reinterpret_cast<const unsigned *>(p));
    else {
        const uint2 v = *reinterpret_cast<const uint2 *>(p);
        c.u[0] = v.x; c.u[1] = v.y;
    }
    return c;
}

// Operands of the NB feature blocks from the words of eight chunks; `below`: how far the block's exponent is below E
template <int NB, typename F, int WORDS>
__device__ __forceinline__ void make_operands(half8 (&o)[NB], const Codes<WORDS> (&c)[CH], int below)
{
    if constexpr (std::is_same<F, Int8Code>::value) {
        const float r = __builtin_ldexpf(1.f, -below);
        const _Float16 s = (_Float16)(r * 32768.f), z = (_Float16)(r * -0.25f);
        const half2q s2 = {s, s}, z2 = {z, z};
        unsigned u[CH][WORDS];
#pragma unroll
        for (int t = 0; t < CH; ++t)
#pragma unroll
            for (int w = 0; w < WORDS; ++w) u[t][w] = c[t].u[w] ^ 0x80808080u;
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int t = 0; t < CH; t += 2) {
                const unsigned sel = 0x0c000c00u | ((unsigned)(4 + i % 4) << 16) | (unsigned)(i % 4);
                const half2q v = __builtin_elementwise_fma(__builtin_bit_cast(half2q, __builtin_amdgcn_perm(u[t + 1][i / 4], u[t][i / 4], sel)), s2, z2);
                o[i][t] = v[0];
                o[i][t + 1] = v[1];
            }
    } else {
        const float scale = __builtin_ldexpf(1.f, 7 - below);
#pragma unroll
        for (int t = 0; t < CH; t += 2)
#pragma unroll
            for (int i = 0; i < NB; i += 2) {             // bytes of features i and i + 1 of both chunks
                const unsigned lo = i % 4, sel = lo | ((4 + lo) << 8) | ((lo + 1) << 16) | ((5 + lo) << 24);
                const unsigned w = __builtin_amdgcn_perm(c[t + 1].u[i / 4], c[t].u[i / 4], sel);
                const half2q a = __builtin_bit_cast(half2q, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, false));
                o[i][t] = a[0];
                o[i][t + 1] = a[1];
                if (i + 1 < NB) {
                    const half2q b = __builtin_bit_cast(half2q, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, true));
                    o[i + 1][t] = b[0];
                    o[i + 1][t + 1] = b[1];
                }
            }
    }
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

template <int D, typename F, typename TQ, bool FUSED, int W, class Lds>
__device__ __forceinline__ void decode_q8_body(const Q8Args &a, const DecPiece &pc, Lds &lds, int wave, int lane)
{
    using S = Q8Shape<D>;
    using U = Unit<F>;
    constexpr int NB = S::NB, NR = S::NR;
    constexpr int row[4] = {S::TEAM ? W : 0, S::TEAM ? 7 - W : 1, 2, 3};
    const int g = lane / 16, nn = lane % 16;
    const int L = pc.L, b = pc.b, bh = pc.bh, hc = pc.h / a.group;
    // pieces begin at blocks of the format, and so do no two waves read one step
    const int p0 = min((pc.k0 + CACHE_BLOCK - 1) & ~(CACHE_BLOCK - 1), L), p1 = pc.k1 >= L ? L : min((pc.k1 + CACHE_BLOCK - 1) & ~(CACHE_BLOCK - 1), L);
    const int share = S::TEAM ? p1 - p0 : ((p1 - p0 + 3) / 4 + STEP - 1) / STEP * STEP;
    const int r0 = __builtin_amdgcn_readfirstlane(min(p0 + (S::TEAM ? 0 : wave * share), p1));
    const int r1 = __builtin_amdgcn_readfirstlane(min(r0 + share, p1));
    const int nsteps = (r1 - r0 + STEP - 1) / STEP;
    const char *Kh = a.K + b * a.sk.batch + hc * a.sk.head, *Vh = a.V + b * a.sv.batch + hc * a.sv.head;
    const int64_t krow = a.sk.seq, vrow = a.sv.seq;
    const unsigned koff = (unsigned)(g * (int)krow + NB * nn), voff = (unsigned)(g * (int)vrow + NB * nn);
    const int8_t *ke = a.ke + (size_t)(b * a.HC + hc) * a.blocks, *ve = a.ve + (size_t)(b * a.HC + hc) * a.blocks;

    struct Step { Codes<S::WORDS> k[CH], v[CH]; };
    auto load = [&](Step &st, int s) {
        const int j0 = r0 + (s < nsteps ? s : 0) * STEP;  // past the end: the first step again, never used
        if (j0 + STEP <= L) {
            const char *kp = Kh + j0 * krow, *vp = Vh + j0 * vrow;
#pragma unroll
            for (int c = 0; c < CH; ++c) st.k[c] = load_codes<NB>(kp + 4 * c * krow + koff);
#pragma unroll
            for (int c = 0; c < CH; ++c) st.v[c] = load_codes<NB>(vp + 4 * c * vrow + voff);
        } else {                                          // rows beyond the sequence: its last row (their weights are 0)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int64_t j = min(j0 + 4 * c + g, L - 1);
                st.k[c] = load_codes<NB>(Kh + j * krow + NB * nn);
                st.v[c] = load_codes<NB>(Vh + j * vrow + NB * nn);
            }
        }
    };

    f32x4 acc[S::NTILES];                                 // (TEAM: the tiles of row blocks row[0] and row[1] only)
    float mu[NR], yv[NR], q[NB];
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
    int EK = EXP_NAN, EV = EXP_NAN;                       // largest exponents of the blocks read
    if (nsteps > 0) {
        Step sa, sb;
        load(sa, 0);
        {
            const TQ *qp = static_cast<const TQ *>(a.out.q) + (size_t)bh * D + NB * nn;
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                if constexpr (sizeof(TQ) == 2) q[i] = bf16_to_f32(qp[i]) * a.cscale;
                else q[i] = qp[i] * a.cscale;
            }
        }
        const int b0 = r0 / CACHE_BLOCK, b1 = (r1 - 1) / CACHE_BLOCK;
        for (int i = b0 + lane; i <= b1; i += 64) {
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
        for (int i = 0; i < NB; ++i) q[i] = __builtin_ldexpf(q[i], EK + U::EXP);

        int ek64 = 0, ev64 = 0;                           // exponents of 64 blocks, one per lane
        auto compute = [&](const Step &st, int s) {
            const int j0 = r0 + s * STEP, at = j0 / CACHE_BLOCK - b0;
            if (at % 64 == 0 && (s == 0 || j0 % CACHE_BLOCK == 0)) {
                const int i = min(b0 + at + lane, b1);
                ek64 = ke[i];
                ev64 = ve[i];
            }
            const int e_k = __builtin_amdgcn_readlane(ek64, at % 64), e_v = __builtin_amdgcn_readlane(ev64, at % 64);
            half8 kh[NB], vh[NB];
            make_operands<NB, F>(kh, st.k, EK - e_k);
            float t[2];
#pragma unroll
            for (int grp = 0; grp < 2; ++grp) {
                float p[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    p[c] = 0.f;
#pragma unroll
                    for (int i = 0; i < NB; ++i) p[c] = fmaf((float)kh[i][4 * grp + c], q[i], p[c]);
                }
                t[grp] = reduce4(p, nn);                  // logit (log2 units) of key 4 (n % 4) + g of the group
                if (e_k == EXP_NAN || e_v == EXP_NAN) t[grp] = NAN;      // (a scalar branch)
                t[grp] = j0 + grp * 16 + 4 * (nn & 3) + g < r1 ? t[grp] : -INFINITY;
            }
            const float top = fmaxf(t[0], t[1]);
            if (__builtin_amdgcn_ballot_w64(top > mref + (U::TOP + 2)) != 0) {
                const float mnew = wave_max_dpp(top) - U::TOP;
                const float alpha = mref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mref - mnew);
                mref = mnew;
                om *= alpha;
#pragma unroll
                for (int i = 0; i < NR; ++i) { mu[i] *= alpha; yv[i] *= alpha; }
                for_tiles([&](int t, bool) { acc[t] *= alpha; });
            }
            mtrue = fmaxf(mtrue, top);
            float w[2];
#pragma unroll
            for (int grp = 0; grp < 2; ++grp) {
                w[grp] = __builtin_amdgcn_exp2f(t[grp] - mref);       // exp2(-inf) = 0 masks the tail
                om += w[grp];
            }
            const float wc[8] = {row_bcast<0>(w[0]), row_bcast<1>(w[0]), row_bcast<2>(w[0]), row_bcast<3>(w[0]),
                                 row_bcast<0>(w[1]), row_bcast<1>(w[1]), row_bcast<2>(w[1]), row_bcast<3>(w[1])};
            make_operands<NB, F>(vh, st.v, EV - e_v);
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                half8 xh, xl;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const float k = (float)kh[row[i]][c];
                    xh[c] = (_Float16)(wc[c] * k);
                    xl[c] = (_Float16)fmaf(wc[c], k, -(float)xh[c]);
                    mu[i] = fmaf(wc[c], k, mu[i]);
                    yv[i] = fmaf(wc[c], (float)vh[row[i]][c], yv[i]);
                }
                auto product = [&](f32x4 &t, const half8 &b) { t = mfma_f16(xh, b, mfma_f16(xl, b, t)); };
#pragma unroll
                for (int J = row[i]; J < NB; ++J) product(acc[upper_tile<NB>(row[i], J)], kh[J]);
#pragma unroll
                for (int J = 0; J < NB; ++J) product(acc[S::NSIG + NB * row[i] + J], vh[J]);
            }
        };
        for (int s = 0; s < nsteps; s += 2) {
            load(sb, s + 1);
            compute(sa, s);
            load(sa, s + 2);
            if (s + 1 < nsteps) compute(sb, s + 1);
        }
        for_tiles([&](int t, bool sigma) {
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][i] = __builtin_ldexpf(acc[t][i], EK + U::EXP + (sigma ? EK : EV) + U::EXP);
        });
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            mu[i] = __builtin_ldexpf(mu[i], EK + U::EXP);
            yv[i] = __builtin_ldexpf(yv[i], EV + U::EXP);
        }
    }

    mtrue = wave_max_dpp(mtrue);
    om += dpp_f<0xB1>(om);
    om += dpp_f<0x4E>(om);
    om = rows_allsum(om);
#pragma unroll
    for (int i = 0; i < NR; ++i) { mu[i] = rows_allsum(mu[i]); yv[i] = rows_allsum(yv[i]); }
    float *R = a.parts + (size_t)pc.rec * S::REC_F;       // this workgroup's record (not FUSED)
    if constexpr (!S::TEAM) {
        finish_workgroup<D, TQ, true, FUSED, S::NBUF>(lds, acc, mu, yv, om, mref, mtrue, R, a.out, bh, wave, lane);
    } else {                                              // every wave's own tiles, relative to the true maximum
        const float f = mref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mref - mtrue);
        float *tiles, *mud, *yvd;
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
            const QueryPart<D> query = load_query<D, TQ, true>(a.out, bh, lane);
            __syncthreads();
            solve_head<D, TQ, true>(lds, a.out, query, bh, wave, lane);
        }
    }
}

template <int D, typename F, typename TQ, bool FUSED>
__global__ __launch_bounds__(NT, D <= 32 ? 4 : (D == 128 && FUSED) ? 1 : 2) void decode_q8_kernel(Q8Args a)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    using S = Q8Shape<D>;
    if constexpr (S::TEAM) {                              // scalar branches; all four waves meet at the same barriers
        __shared__ __align__(16) unsigned char raw[FUSED ? sizeof(HeadLds<D, 1, 1>) : 16];
        HeadLds<D, 1, 1> &lds = *reinterpret_cast<HeadLds<D, 1, 1> *>(raw);
        for_pieces<FUSED>(a.split, [&](const DecPiece &pc) {
            if (wave == 0) decode_q8_body<D, F, TQ, FUSED, 0>(a, pc, lds, wave, piece_lane());
            else if (wave == 1) decode_q8_body<D, F, TQ, FUSED, 1>(a, pc, lds, wave, piece_lane());
            else if (wave == 2) decode_q8_body<D, F, TQ, FUSED, 2>(a, pc, lds, wave, piece_lane());
            else decode_q8_body<D, F, TQ, FUSED, 3>(a, pc, lds, wave, piece_lane());
        });
    } else {
        __shared__ HeadLds<D, S::NBUF, 4> lds;
        for_pieces<FUSED>(a.split, [&](const DecPiece &pc) { decode_q8_body<D, F, TQ, FUSED, 0>(a, pc, lds, wave, piece_lane()); });
    }
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

template <int D, typename F, typename TQ>
__global__ __launch_bounds__(NT) void short_heads_kernel(Q8Args a, float scale)
{
    __shared__ dual::DualShared<D, DUAL_MAX_KEYS> sm;
    if (a.out.out_bf16) short_head<D, F, TQ, bf16_t>(sm, a, scale, blockIdx.x);
    else short_head<D, F, TQ, float>(sm, a, scale, blockIdx.x);
}

// Merge of the records, one workgroup per head, and behind them one per head for short sequences; which of the two writes the head follows from
// its length
template <int D, typename F, typename TQ>
__global__ __launch_bounds__(NT, D == 128 ? 1 : 2) void merge_q8_kernel(Q8Args a, float scale, int heads)
{
    using Dual = dual::DualShared<D, DUAL_MAX_KEYS>;
    constexpr size_t LDS_B = sizeof(HeadLds<D, 1, 1>) > sizeof(Dual) ? sizeof(HeadLds<D, 1, 1>) : sizeof(Dual);
    __shared__ __align__(16) unsigned char raw[LDS_B];
    if ((int)blockIdx.x >= heads) {
        if (a.out.out_bf16) short_head<D, F, TQ, bf16_t>(*reinterpret_cast<Dual *>(raw), a, scale, blockIdx.x - heads);
        else short_head<D, F, TQ, float>(*reinterpret_cast<Dual *>(raw), a, scale, blockIdx.x - heads);
        return;
    }
    if (seq_len(a.split, blockIdx.x / a.split.H) <= DUAL_MAX_KEYS) return;
    merge_head<D, TQ, true>(*reinterpret_cast<HeadLds<D, 1, 1> *>(raw), a.split, a.out, a.parts, blockIdx.x);
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
    if (c.L_max <= DUAL_MAX_KEYS) {
        a.split = DecSplit{p.seqlens, c.B, p.H, c.L_max, 1, 0, 0, 0, 0};
        stage_mark(p.stream, "decode_q8_short");
        hipLaunchKernelGGL((short_heads_kernel<D, F, TQ>), dim3(bh), dim3(NT), 0, p.stream, a, p.scale);
        return hipGetLastError();
    }
    const size_t records = q8_records<D>(c.B, p.H, c.L_max);
    const bool scratch = p.ws != nullptr && (reinterpret_cast<uintptr_t>(p.ws) & 255u) == 0 && p.ws_bytes >= records * S::REC_F * sizeof(float);
    const int ns = scratch ? q8_nsplit<D>(bh, c.L_max) : 1;
    a.split = choose_split(cut, ns, scratch ? records : 0, S::SLOTS, 2 * CACHE_BLOCK, S::KEYS_MIN, S::MAX_SPLIT);
    if (a.split.nsplit == 1 && a.split.slots == 0) {
        stage_mark(p.stream, "decode_q8");
        hipLaunchKernelGGL((decode_q8_kernel<D, F, TQ, true>), dim3(1, bh), dim3(NT), 0, p.stream, a);
        if (p.seqlens != nullptr) hipLaunchKernelGGL((short_heads_kernel<D, F, TQ>), dim3(bh), dim3(NT), 0, p.stream, a, p.scale);
    } else {
        stage_mark(p.stream, "decode_q8_partial");
        hipLaunchKernelGGL((decode_q8_kernel<D, F, TQ, false>), a.split.slots ? dim3(a.split.slots, p.H) : dim3(a.split.nsplit, bh), dim3(NT), 0, p.stream, a);
        stage_mark(p.stream, "decode_q8_merge");
        hipLaunchKernelGGL((merge_q8_kernel<D, F, TQ>), dim3(p.seqlens ? 2 * bh : bh), dim3(NT), 0, p.stream, a, p.scale, bh);
    }
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
