// llla_cache_scores: the share of every query's kernel weight that each cached row has, summed over the queries.
//
// All queries that read a cache head (its group of query heads, nq of each) are the rows r of one matrix: logits T = K Q^T on bf16 matrix
// instructions, keys as rows of a tile and queries as columns, so that the sums over keys (omega of a query) and over queries (a row's share)
// are sums in a lane with one exchange at the end.  Two passes, because a share needs its query's omega: statistics (largest logit and sum of
// weights per query), then shares.  Codes and bf16 numbers are operands as they are; fp32 is split into three bf16 (24 bits), six products.
//   few queries (decode): the first pass is bound by the cache's traffic; it leaves the logits, and the second reads those
//   many (prompts): both passes form the logits; what bounds them is one exponential per logit and pass
#include <algorithm>

#include "llla_cache.hpp"
#include "llla_mfma_common.hpp"
#include "llla_mfma_solve64.hpp"

namespace llla {
namespace {

using namespace mfma;

constexpr int NT = 256, NW = NT / 64;

template <typename T> struct RowType;                     // how a row of the cache or a query becomes operands
template <> struct RowType<float> { static constexpr int SIZE = 4, TERMS = 3; };
template <> struct RowType<bf16_t> { static constexpr int SIZE = 2, TERMS = 1; };
template <> struct RowType<Int8Code> { static constexpr int SIZE = 1, TERMS = 1; };
template <> struct RowType<E4m3Code> { static constexpr int SIZE = 1, TERMS = 1; };

// Lane (g, n) holds features g D / 4 .. of row n, eight to a step of 32 (at d = 16 four, the others zero): whole rows in loads of up to
// sixteen bytes.  Any order of the features will do, as long as both operands have it.
template <int D, typename T>
struct Operand {
    static constexpr int CH = D < 32 ? 1 : D / 32, TERMS = RowType<T>::TERMS;
    bf16x8 v[CH][TERMS];
};

template <int D, typename T>
__device__ __forceinline__ void load_operand(Operand<D, T> &o, const char *row, int g)
{
    constexpr int PER = D / 4, SIZE = RowType<T>::SIZE, BYTES = PER * SIZE, CH = Operand<D, T>::CH;
    constexpr int N = PER < 8 ? PER : 8;                  // features of a step
    unsigned w[BYTES / 4];
    const char *p = row + g * BYTES;
    if constexpr (BYTES == 4) w[0] = *reinterpret_cast<const unsigned *>(p);
    else if constexpr (BYTES == 8) {
        const uint2 v = *reinterpret_cast<const uint2 *>(p);
        w[0] = v.x; w[1] = v.y;
    } else {
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) {
            const uint4 v = reinterpret_cast<const uint4 *>(p)[i];
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        if constexpr (std::is_same<T, bf16_t>::value) {
            unsigned u[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < N / 2; ++i) u[i] = w[4 * c + i];
            o.v[c][0] = __builtin_bit_cast(bf16x8, u);
        } else {
            float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if constexpr (SIZE == 4) {
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = __uint_as_float(w[8 * c + i]);
                split3_bf16(x, o.v[c][0], o.v[c][1], o.v[c][2]);
            } else {
#pragma unroll
                for (int i = 0; i < N / 4; ++i) {
                    float y[4];
                    decode4<T>(w[2 * c + i], y);
#pragma unroll
                    for (int t = 0; t < 4; ++t) x[4 * i + t] = y[t];
                }
                unsigned u[4];                            // (exact: the upper halves are the numbers)
#pragma unroll
                for (int i = 0; i < 4; ++i) u[i] = __builtin_amdgcn_perm(__float_as_uint(x[2 * i + 1]), __float_as_uint(x[2 * i]), 0x07060302u);
                o.v[c][0] = __builtin_bit_cast(bf16x8, u);
            }
        }
    }
}

// 16 keys x 16 queries: lane (g, n), register t: key 4 g + t, query n
template <int D, typename TK, typename TQ>
__device__ __forceinline__ f32x4 logits(const Operand<D, TK> &k, const Operand<D, TQ> &q)
{
    f32x4 t = {0.f, 0.f, 0.f, 0.f};
    constexpr int CH = Operand<D, TK>::CH, PK = Operand<D, TK>::TERMS, PQ = Operand<D, TQ>::TERMS;
#pragma unroll
    for (int s = PK + PQ - 2; s >= 0; --s)                // small terms first; what is below 2^-24 is left out
#pragma unroll
        for (int i = 0; i < PK; ++i) {
            const int j = s - i;
            if (j < 0 || j >= PQ || s > 2) continue;
#pragma unroll
            for (int c = 0; c < CH; ++c) t = mfma_bf16(k.v[c][i], q.v[c][j], t);
        }
    return t;
}

struct ScoresArgs {
    const char *Q, *K;
    llla_strides sq, sk;               // in bytes
    const int8_t *ke;
    float *scores;
    const int32_t *seqlens;
    int HC, group, nq, M, L_max;       // M: queries of a cache head
    int splits;                        // parts of the keys, in the statistics of few queries
    float cscale;                      // log2(e) * scale
    float *stats;                      // [B HC][splits][M] pairs (largest logit, sum), or with one part [B HC][M] log2 of the sums
    float *logits;                     // [B HC][M][pitch], or nullptr
    int64_t pitch;
};

struct Head { int b, h, len; };
__device__ __forceinline__ Head head_of(const ScoresArgs &a, int bh)
{
    Head x;
    x.b = bh / a.HC;
    x.h = bh % a.HC;
    x.len = cache_length(a.seqlens, x.b, a.L_max);
    return x;
}

__device__ __forceinline__ const char *query_row(const ScoresArgs &a, const Head &x, int r)
{
    return a.Q + x.b * a.sq.batch + (int64_t)(x.h * a.group + r / a.nq) * a.sq.head + (int64_t)(r % a.nq) * a.sq.seq;
}
// keys that query r sees: slots below this
__device__ __forceinline__ int limit_of(const ScoresArgs &a, const Head &x, int r) { return r < a.M ? x.len - a.nq + r % a.nq + 1 : 0; }

// the block's power of two, times the scale of the logits
template <typename TK>
__device__ __forceinline__ float tile_scale(const ScoresArgs &a, int bh, int key)
{
    if constexpr (RowType<TK>::SIZE > 1) return a.cscale;
    else {
        const int e = a.ke[(size_t)bh * cache_blocks(a.L_max) + key / CACHE_BLOCK];
        return e == EXP_NAN ? NAN : __builtin_ldexpf(a.cscale, e);
    }
}

// largest logit m and sum of weights l relative to it, of two sets of keys
__device__ __forceinline__ void join(float &m, float &l, float m2, float l2)
{
    const float top = fmaxf(m, m2), ref = top == -INFINITY ? 0.f : top;
    l = l * __builtin_amdgcn_exp2f(m - ref) + l2 * __builtin_amdgcn_exp2f(m2 - ref);
    m = top;
}

// Statistics of 16 RT queries per wave.  ROWS: the waves of a workgroup have queries of their own and walk through the same keys; otherwise
// they share the queries and have parts of the keys.
template <int D, typename TK, typename TQ, int RT, bool ROWS>
__global__ __launch_bounds__(NT) void stats_kernel(ScoresArgs a)
{
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), g = lane / 16, n = lane % 16;
    const int bh = blockIdx.y;
    const Head x = head_of(a, bh);
    const int rb = ROWS ? (int)(gridDim.x - 1 - blockIdx.x) * NW + wave : 0, r0 = rb * 16 * RT;      // (the last queries see most: first)
    if (r0 >= a.M) return;
    int k0 = 0, k1 = x.len;
    if (!ROWS) {
        const int part = ((x.len + a.splits - 1) / a.splits + 63) & ~63, s = blockIdx.x * NW + wave;
        k0 = min((int64_t)s * part, (int64_t)x.len);
        k1 = min(k0 + part, x.len);
    }
    Operand<D, TQ> q[RT];
    int lim[RT];
    float m[RT], l[RT];
    int most = 0;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int r = r0 + 16 * i + n;
        load_operand<D, TQ>(q[i], query_row(a, x, min(r, a.M - 1)), g);
        lim[i] = limit_of(a, x, r);
        most = max(most, lim[i]);
        m[i] = -INFINITY;
        l[i] = 0.f;
    }
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) most = max(most, __shfl_xor(most, off));
    k1 = min(k1, __builtin_amdgcn_readfirstlane(most));
    const char *Kh = a.K + x.b * a.sk.batch + x.h * a.sk.head;
    for (int j0 = k0; j0 < k1; j0 += 64) {
        f32x4 t[4][RT];
        const float c = tile_scale<TK>(a, bh, j0);
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
            Operand<D, TK> k;
            load_operand<D, TK>(k, Kh + (int64_t)min(j0 + 16 * kt + n, x.len - 1) * a.sk.seq, g);
#pragma unroll
            for (int i = 0; i < RT; ++i) t[kt][i] = logits<D, TK, TQ>(k, q[i]);
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            float top = m[i];
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = j0 + 16 * kt + 4 * g + e;
                    t[kt][i][e] = key < min(lim[i], k1) ? c * t[kt][i][e] : -INFINITY;
                    top = fmaxf(top, t[kt][i][e]);
                }
            const float ref = top == -INFINITY ? 0.f : top;
            float s = l[i] * __builtin_amdgcn_exp2f(m[i] - ref);
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                for (int e = 0; e < 4; ++e) s += __builtin_amdgcn_exp2f(t[kt][i][e] - ref);
            l[i] = s;
            m[i] = top;
            if (!ROWS && a.logits != nullptr && r0 + 16 * i + n < a.M) {
                float *row = a.logits + ((size_t)bh * a.M + r0 + 16 * i + n) * a.pitch + j0 + 4 * g;
#pragma unroll
                for (int kt = 0; kt < 4; ++kt) *reinterpret_cast<f32x4 *>(row + 16 * kt) = t[kt][i];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        join(m[i], l[i], __shfl_xor(m[i], 16), __shfl_xor(l[i], 16));
        join(m[i], l[i], __shfl_xor(m[i], 32), __shfl_xor(l[i], 32));
        const int r = r0 + 16 * i + n;
        if (g == 0 && r < a.M) {
            if (ROWS) {
                a.stats[(size_t)bh * a.M + r] = l[i] == 0.f ? INFINITY : m[i] + __builtin_amdgcn_logf(l[i]);
            } else {
                const size_t at = ((size_t)bh * a.splits + blockIdx.x * NW + wave) * a.M + r;
                a.stats[2 * at] = m[i];
                a.stats[2 * at + 1] = l[i];
            }
        }
    }
}

constexpr int FEW = 64;                                   // queries at most whose keys are cut into parts

// log2 of the sums of weights of a head's few queries, from its parts
__device__ __forceinline__ void merge_stats(const ScoresArgs &a, int bh, float (&lse)[FEW])
{
    // four threads per query, each every fourth part
    const int r = threadIdx.x / 4, sub = threadIdx.x % 4;
    float m = -INFINITY, l = 0.f;
    if (r < a.M)
        for (int s = sub; s < a.splits; s += 4) {
            const size_t at = ((size_t)bh * a.splits + s) * a.M + r;
            join(m, l, a.stats[2 * at], a.stats[2 * at + 1]);
        }
    join(m, l, __shfl_xor(m, 1), __shfl_xor(l, 1));
    join(m, l, __shfl_xor(m, 2), __shfl_xor(l, 2));
    if (sub == 0 && r < a.M) lse[r] = l == 0.f ? INFINITY : m + __builtin_amdgcn_logf(l);
    __syncthreads();
}

// Shares from stored logits: four keys per thread
__global__ __launch_bounds__(NT) void stored_shares_kernel(ScoresArgs a)
{
    __shared__ float lse[FEW];
    const int bh = blockIdx.y, len = cache_length(a.seqlens, bh / a.HC, a.L_max), j = (blockIdx.x * NT + threadIdx.x) * 4;
    if ((int)blockIdx.x * NT * 4 >= len) return;
    merge_stats(a, bh, lse);
    if (j >= len) return;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    for (int r = 0; r < a.M; ++r) {
        // (keys behind the last one that any query sees have no logits)
        const int lim = min(len, len - a.nq + r % a.nq + 1);
        const f32x4 t = *reinterpret_cast<const f32x4 *>(a.logits + ((size_t)bh * a.M + r) * a.pitch + j);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += j + e < lim ? __builtin_amdgcn_exp2f(t[e] - lse[r]) : 0.f;
    }
    float *out = a.scores + (size_t)bh * a.L_max + j;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (j + e < len) out[e] += s[e];
}

// Shares of 64 keys per workgroup, whose waves take every fourth tile of the queries; summed in a fixed order
template <int D, typename TK, typename TQ>
__global__ __launch_bounds__(NT) void shares_kernel(ScoresArgs a)
{
    __shared__ float lse[FEW];
    __shared__ float part[NW][64];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), g = lane / 16, n = lane % 16;
    const int bh = blockIdx.y, j0 = blockIdx.x * 64;
    const Head x = head_of(a, bh);
    if (j0 >= x.len) return;
    if (a.splits > 0) merge_stats(a, bh, lse);
    const char *Kh = a.K + x.b * a.sk.batch + x.h * a.sk.head;
    Operand<D, TK> k[4];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) load_operand<D, TK>(k[kt], Kh + (int64_t)min(j0 + 16 * kt + n, x.len - 1) * a.sk.seq, g);
    const float c = tile_scale<TK>(a, bh, j0);
    f32x4 s[4];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) s[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int r0 = 16 * wave; r0 < a.M; r0 += 16 * NW) {
        const int r = r0 + n, lim = limit_of(a, x, r);
        if (__builtin_amdgcn_ballot_w64(lim > j0) == 0) continue;
        Operand<D, TQ> q;
        load_operand<D, TQ>(q, query_row(a, x, min(r, a.M - 1)), g);
        const float ref = r >= a.M ? INFINITY : a.splits > 0 ? lse[r] : a.stats[(size_t)bh * a.M + r];
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
            const f32x4 t = logits<D, TK, TQ>(k[kt], q);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = __builtin_amdgcn_exp2f(fmaf(c, t[e], -ref));
                s[kt][e] += j0 + 16 * kt + 4 * g + e < lim ? p : 0.f;
            }
        }
    }
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float v = row_allsum(s[kt][e]);
            if (n == 0) part[wave][16 * kt + 4 * g + e] = v;
        }
    __syncthreads();
    const int j = threadIdx.x;
    if (j < 64 && j0 + j < x.len) a.scores[(size_t)bh * a.L_max + j0 + j] += (part[0][j] + part[1][j]) + (part[2][j] + part[3][j]);
}

// How a call is cut
struct ScoresPlan {
    int M, splits;             // splits == 0: the waves have queries of their own
    bool stored;
    int64_t pitch;
    size_t stats_bytes, bytes;
};

ScoresPlan scores_plan(const llla_cache &c, int H, int nq)
{
    ScoresPlan p{};
    p.M = H / c.H * nq;
    const int heads = c.B * c.H, size = c.type == LLLA_F32 ? 4 : c.type == LLLA_BF16 ? 2 : 1;
    if (p.M <= FEW) {
        // enough workgroups for the GPU, each wave with at least 256 keys
        const int wgs = std::max(1, std::min((2048 + heads - 1) / heads, (c.L_max + 1023) / 1024));
        p.splits = NW * wgs;
        // a logit is written and read, a row of the cache would be read a second time
        p.stored = 8 * p.M <= c.d * size;
    }
    p.pitch = p.stored ? (int64_t)(c.L_max + 63) / 64 * 64 : 0;
    p.stats_bytes = round_up((size_t)heads * p.M * (p.splits ? 2 * p.splits : 1) * sizeof(float), 256);
    p.bytes = p.stats_bytes + round_up((size_t)heads * p.M * p.pitch * sizeof(float), 256);
    return p;
}

template <int D, typename TK, typename TQ>
hipError_t launch_scores(const ScoresProblem &p)
{
    const llla_cache &c = p.c;
    const ScoresPlan plan = scores_plan(c, p.H, p.nq);
    constexpr int KS = RowType<TK>::SIZE, QS = RowType<TQ>::SIZE, RT = QS == 4 ? 2 : 4;
    ScoresArgs a{};
    a.Q = static_cast<const char *>(p.Q);
    a.K = static_cast<const char *>(c.K);
    a.sq = llla_strides{p.sq.batch * QS, p.sq.head * QS, p.sq.seq * QS};
    a.sk = llla_strides{c.sk.batch * KS, c.sk.head * KS, c.sk.seq * KS};
    a.ke = c.k_exp;
    a.scores = c.scores;
    a.seqlens = p.seqlens;
    a.HC = c.H; a.group = p.H / c.H; a.nq = p.nq; a.M = plan.M; a.L_max = c.L_max;
    a.splits = plan.splits;
    a.cscale = p.scale * LOG2E;
    a.stats = static_cast<float *>(p.ws);
    a.logits = plan.stored ? reinterpret_cast<float *>(static_cast<char *>(p.ws) + plan.stats_bytes) : nullptr;
    a.pitch = plan.pitch;
    const int heads = c.B * c.H;
    if (plan.splits > 0) {
        const dim3 grid(plan.splits / NW, heads);
        if (plan.M <= 16) hipLaunchKernelGGL((stats_kernel<D, TK, TQ, 1, false>), grid, dim3(NT), 0, p.stream, a);
        else if (plan.M <= 32) hipLaunchKernelGGL((stats_kernel<D, TK, TQ, 2, false>), grid, dim3(NT), 0, p.stream, a);
        else hipLaunchKernelGGL((stats_kernel<D, TK, TQ, 4, false>), grid, dim3(NT), 0, p.stream, a);
    } else {
        const int rows = 16 * RT * NW;
        hipLaunchKernelGGL((stats_kernel<D, TK, TQ, RT, true>), dim3((plan.M + rows - 1) / rows, heads), dim3(NT), 0, p.stream, a);
    }
    if (plan.stored) hipLaunchKernelGGL(stored_shares_kernel, dim3((c.L_max + 4 * NT - 1) / (4 * NT), heads), dim3(NT), 0, p.stream, a);
    else hipLaunchKernelGGL((shares_kernel<D, TK, TQ>), dim3((c.L_max + 63) / 64, heads), dim3(NT), 0, p.stream, a);
    return hipGetLastError();
}

template <int D>
hipError_t scores_by_type(const ScoresProblem &p)
{
    const bool f32 = p.in == LLLA_F32;
    switch (p.c.type) {
        case LLLA_I8: return f32 ? launch_scores<D, Int8Code, float>(p) : launch_scores<D, Int8Code, bf16_t>(p);
        case LLLA_E4M3: return f32 ? launch_scores<D, E4m3Code, float>(p) : launch_scores<D, E4m3Code, bf16_t>(p);
        case LLLA_BF16: return launch_scores<D, bf16_t, bf16_t>(p);
        default: return launch_scores<D, float, float>(p);
    }
}

}  // namespace

size_t cache_scores_workspace_bytes(const llla_cache &c, int H, int nq, llla_dtype) { return scores_plan(c, H, nq).bytes; }

hipError_t cache_scores(const ScoresProblem &p)
{
    switch (p.c.d) {
        case 16: return scores_by_type<16>(p);
        case 32: return scores_by_type<32>(p);
        case 64: return scores_by_type<64>(p);
        case 128: return scores_by_type<128>(p);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace llla
