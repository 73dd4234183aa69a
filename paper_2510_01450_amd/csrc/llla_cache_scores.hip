// llla_cache_scores: the share of every query's kernel weight that each cached row has, summed over the queries.
//
// All queries that read a cache head (its group of query heads, nq of each) are the rows r of one matrix: logits T = K Q^T on bf16 matrix
// instructions, keys as rows of a tile and queries as columns, so that the sums over keys (omega of a query) and over queries (a row's share)
// are sums in a lane with one exchange at the end.  Two passes, because a share needs its query's omega: statistics (largest logit and sum of
// weights per query), then shares.  Codes and bf16 numbers are operands as they are; fp32 is split into three bf16 (24 bits), six products.
//   few queries (decode): the first pass is bound by the cache's traffic; it leaves the logits, and the second reads those
//     (512 heads x 32768 int8 keys 220 + 32 us, 4.9 TB/s)
//   many (prompts): both passes form the logits; per logit and pass one exponential, one multiply-add and one addition on the vector port
//     (32 heads, 4096 queries over 4096 bf16 keys: 82 + 88 us, 3.2 logits per ps and pass; the least that those three instructions take, 17
//     cycles of a wave as measured, is 29 us a pass; rows come from L2)
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

// Lane (g, n) holds a quarter of row n's features, eight to a step of 32 (at d = 16 four, the others zero).  Any order of the features will do, as long as
// both operands have it: groups of the sixteen bytes of a key go to the four lanes in turn, so that a load reads 64 consecutive bytes of every row (with
// a lane's bytes consecutive, 128 of an fp32 row at d = 128, lines that were not to be kept were fetched more than once: 14 heads of 4006 rows 27 us).
template <int D, typename T>
struct Operand {
    static constexpr int CH = D < 32 ? 1 : D / 32, TERMS = RowType<T>::TERMS;
    bf16x8 v[CH][TERMS];
};

// a lane's part of a row as it lies in memory
template <int D, typename T>
struct Words {
    static constexpr int BYTES = D / 4 * RowType<T>::SIZE;
    unsigned w[BYTES / 4];
};

// features of a group
template <int D, typename TK> constexpr int GROUP = 16 / RowType<TK>::SIZE < D / 4 ? 16 / RowType<TK>::SIZE : D / 4;

// of a key or, T = TQ, a query to keys of type TK; ONCE: not to be kept in the caches
template <int D, typename TK, typename T, bool ONCE = false>
__device__ __forceinline__ Words<D, T> load_words(const char *row, int g)
{
    constexpr int G = GROUP<D, TK>, BYTES = G * RowType<T>::SIZE, N = BYTES < 16 ? BYTES / 4 : 4, LOADS = BYTES / 4 / N;
    typedef unsigned part __attribute__((ext_vector_type(N)));
    Words<D, T> o;
#pragma unroll
    for (int i = 0; i < D / 4 / G; ++i) {
        const part *p = reinterpret_cast<const part *>(row + (4 * i + g) * BYTES);
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            const part v = ONCE ? __builtin_nontemporal_load(p + k) : p[k];
#pragma unroll
            for (int e = 0; e < N; ++e) o.w[N * (LOADS * i + k) + e] = v[e];
        }
    }
    return o;
}

template <int D, typename T>
__device__ __forceinline__ void make_operand(Operand<D, T> &o, const Words<D, T> &in)
{
    constexpr int PER = D / 4, SIZE = RowType<T>::SIZE, CH = Operand<D, T>::CH;
    constexpr int N = PER < 8 ? PER : 8;                  // features of a step
    const auto &w = in.w;
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

// the negative row, for a scale below zero: the largest logit is then that of the largest product too
template <int D, typename T>
__device__ __forceinline__ void negate(Operand<D, T> &o)
{
#pragma unroll
    for (int c = 0; c < Operand<D, T>::CH; ++c)
#pragma unroll
        for (int i = 0; i < Operand<D, T>::TERMS; ++i) {
            typedef unsigned u32x4q __attribute__((ext_vector_type(4)));
            o.v[c][i] = __builtin_bit_cast(bf16x8, (u32x4q)(__builtin_bit_cast(u32x4q, o.v[c][i]) ^ 0x80008000u));
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
    int splits;                        // parts of the keys in the statistics
    int blocks;                        // workgroups of queries there (0: a workgroup's waves share the queries)
    float cscale;                      // log2(e) |scale|
    int negative;                      // scale < 0
    float *stats;                      // [B HC][splits][M] pairs (largest logit, sum)
    float *lse;                        // [B HC][M] log2 of the sums of weights, or nullptr: merged by who needs them
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

// Query r of a cache head: query i of query head h; beyond the last one the last (it sees nothing)
struct Query {
    int h, i;
    bool real;
    __device__ Query(const ScoresArgs &a, int r) : h(min(r, a.M - 1) / a.nq), i(min(r, a.M - 1) % a.nq), real(r < a.M) {}
    __device__ const char *row(const ScoresArgs &a, const Head &x) const
    {
        return a.Q + x.b * a.sq.batch + (int64_t)(x.h * a.group + h) * a.sq.head + (int64_t)i * a.sq.seq;
    }
    // keys that it sees: slots below this
    __device__ int limit(const ScoresArgs &a, const Head &x) const { return real ? x.len - a.nq + i + 1 : 0; }
};

template <int D, typename TQ>
__device__ __forceinline__ void query_operand(Operand<D, TQ> &o, const ScoresArgs &a, const Words<D, TQ> &w)
{
    make_operand<D, TQ>(o, w);
    if (a.negative) negate<D, TQ>(o);                     // (a scalar branch)
}

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

// 256 registers for a wave (matrix results then stay where vector instructions read them), or all 512 where operands of three terms need them
template <int D, typename TK, typename TQ, int RT>
struct RegisterFile {
    static constexpr int NEED = D / 32 * 4 * (RT * RowType<TQ>::TERMS + 4 * RowType<TK>::TERMS);
    static constexpr int WAVES = NEED > 128 ? 1 : 2;
};

// Consecutive workgroups get heads in turn: an XCD, which takes each eighth of them, then has the rows of an eighth of the heads in its L2 (32 heads, 4096 queries
// over 4096 bf16 keys 229 -> 174 us), and parts that see many keys and few alike.  (Grids of 2^32 and more as they are.)
__device__ __forceinline__ void by_head(int &bh, int &at)
{
    const uint64_t all = (uint64_t)gridDim.x * gridDim.y;
    if (all >> 32) return;
    const unsigned id = blockIdx.y * gridDim.x + blockIdx.x, heads = gridDim.y;
    at = (int)(id / heads);
    bh = (int)(id - (unsigned)at * heads);
}

__device__ __forceinline__ int wave_min(int x)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x = min(x, __shfl_xor(x, off));
    return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ int wave_max(int x)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x = max(x, __shfl_xor(x, off));
    return __builtin_amdgcn_readfirstlane(x);
}

// Statistics of 16 RT queries per wave.  ROWS: the waves of a workgroup have queries of their own and walk through the same keys; otherwise
// they share the queries and have parts of the keys.
// Per logit one fused multiply-add, one exponential and one addition.  A sum of weights relative to any logit of its keys is as good as one
// relative to the largest while it stays below FAR: the reference is the first block's largest, and is raised by the block that passes FAR.
// Masks only in blocks that some query does not see whole.  Rows are requested PF tiles of 16 keys ahead.
constexpr float FAR = 0x1p64f;

template <int D, typename TK, typename TQ, int RT, bool ROWS>
__global__ __launch_bounds__(NT, (RegisterFile<D, TK, TQ, RT>::WAVES)) void stats_kernel(ScoresArgs a)
{
    constexpr int PF = Words<D, TK>::BYTES > 64 ? 1 : 4;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), g = lane / 16, n = lane % 16;
    int bh = blockIdx.y, at = blockIdx.x;
    if constexpr (ROWS) by_head(bh, at);
    const Head x = head_of(a, bh);
    // (the last queries see most: first)
    const int r0 = ROWS ? ((a.blocks - 1 - at % a.blocks) * NW + wave) * 16 * RT : 0, part = ROWS ? at / a.blocks : at * NW + wave;
    if (r0 >= a.M) return;
    const int each = ((x.len + a.splits - 1) / a.splits + 63) & ~63;
    const int k0 = (int)min((int64_t)part * each, (int64_t)x.len);
    Operand<D, TQ> q[RT];
    int lim[RT], most = 0, least = INT32_MAX;
    float m[RT], l[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const Query r(a, r0 + 16 * i + n);
        query_operand<D, TQ>(q[i], a, load_words<D, TK, TQ>(r.row(a, x), g));
        lim[i] = r.limit(a, x);
        most = max(most, lim[i]);
        least = min(least, r.real ? lim[i] : INT32_MAX);
        m[i] = -INFINITY;
        l[i] = 0.f;
    }
    const int k1 = min(min(k0 + each, x.len), wave_max(most));
    least = min(wave_min(least), k1);
    const char *Kh = a.K + x.b * a.sk.batch + x.h * a.sk.head;
    // A tile's rows from a scalar base: one vector minimum for the rows behind the last (row strides are below 2^27 bytes)
    const unsigned far_row = (unsigned)n * (unsigned)a.sk.seq;
    auto load = [&](int j) {
        const int at = min(j, x.len - 1);
        const unsigned last = (unsigned)min(15, x.len - 1 - at) * (unsigned)a.sk.seq;
        return load_words<D, TK, TK, !ROWS && RT == 1>(Kh + at * a.sk.seq + min(far_row, last), g);
    };
    if (k0 < k1) {
        Words<D, TK> ahead[PF];
#pragma unroll
        for (int i = 0; i < PF; ++i) ahead[i] = load(k0 + 16 * i);
        for (int j0 = k0; j0 < k1; j0 += 64) {
            f32x4 t[4][RT];
            const float c = tile_scale<TK>(a, bh, j0);
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
                Operand<D, TK> k;
                make_operand<D, TK>(k, ahead[kt % PF]);
                ahead[kt % PF] = load(j0 + 16 * (kt + PF));
#pragma unroll
                for (int i = 0; i < RT; ++i) t[kt][i] = logits<D, TK, TQ>(k, q[i]);
            }
            const bool masked = j0 + 64 > least;          // (scalar)
            if (masked) {
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) t[kt][i][e] = j0 + 16 * kt + 4 * g + e < min(lim[i], k1) ? c * t[kt][i][e] : -INFINITY;
            }
            const float cc = masked ? 1.f : c;
            float sum[RT];
            bool far = j0 == k0;
            if (!far) {
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    const float ref = m[i];
                    float s = 0.f;
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s += __builtin_amdgcn_exp2f(fmaf(cc, t[kt][i][e], -ref));
                    sum[i] = s;
                    far = far || !(s < FAR);
                }
                far = __builtin_amdgcn_ballot_w64(far) != 0;
            }
            if (far) {
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    float top = -INFINITY;
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                        for (int e = 0; e < 4; e += 2) top = fmaxf(fmaxf(t[kt][i][e], t[kt][i][e + 1]), top);
                    top = fmaxf(m[i], cc * top);
                    const float ref = top == -INFINITY ? 0.f : top;
                    float s = 0.f;
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s += __builtin_amdgcn_exp2f(fmaf(cc, t[kt][i][e], -ref));
                    l[i] = l[i] * __builtin_amdgcn_exp2f(m[i] - ref) + s;
                    m[i] = top;
                }
            } else {
#pragma unroll
                for (int i = 0; i < RT; ++i) l[i] += sum[i];
            }
            if (!ROWS && a.logits != nullptr) {
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    if (r0 + 16 * i + n >= a.M) continue;
                    float *row = a.logits + ((size_t)bh * a.M + r0 + 16 * i + n) * a.pitch + j0 + 4 * g;
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt) *reinterpret_cast<f32x4 *>(row + 16 * kt) = cc * t[kt][i];
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        join(m[i], l[i], __shfl_xor(m[i], 16), __shfl_xor(l[i], 16));
        join(m[i], l[i], __shfl_xor(m[i], 32), __shfl_xor(l[i], 32));
        const int r = r0 + 16 * i + n;
        if (g == 0 && r < a.M) {
            if (ROWS && a.splits == 1) {
                a.lse[(size_t)bh * a.M + r] = l[i] == 0.f ? INFINITY : m[i] + __builtin_amdgcn_logf(l[i]);
            } else {
                const size_t at = ((size_t)bh * a.splits + part) * a.M + r;
                a.stats[2 * at] = m[i];
                a.stats[2 * at + 1] = l[i];
            }
        }
    }
}

constexpr int FEW = 64;                                   // queries at most that a workgroup's waves share in the statistics

// log2 of the sum of weights of query r, from its parts; by `width` neighbouring threads (a power of two up to 64)
__device__ __forceinline__ float merged(const ScoresArgs &a, int bh, int r, int sub, int width)
{
    float m = -INFINITY, l = 0.f;
    if (r < a.M)
        for (int s = sub; s < a.splits; s += width) {
            const size_t at = ((size_t)bh * a.splits + s) * a.M + r;
            join(m, l, a.stats[2 * at], a.stats[2 * at + 1]);
        }
    for (int off = 1; off < width; off *= 2) join(m, l, __shfl_xor(m, off), __shfl_xor(l, off));
    return l == 0.f ? INFINITY : m + __builtin_amdgcn_logf(l);
}

// of a head's few queries, in LDS
__device__ __forceinline__ void merge_few(const ScoresArgs &a, int bh, float (&lse)[FEW])
{
    const int shift = a.M <= NT / 64 ? 6 : a.M <= NT / 16 ? 4 : 2, r = threadIdx.x >> shift, sub = threadIdx.x & ((1 << shift) - 1);
    const float v = merged(a, bh, r, sub, 1 << shift);
    if (sub == 0) lse[r] = v;
    __syncthreads();
}

__global__ __launch_bounds__(NT) void merge_stats_kernel(ScoresArgs a)
{
    const int r = blockIdx.x * (NT / 4) + threadIdx.x / 4;
    const float v = merged(a, blockIdx.y, r, threadIdx.x % 4, 4);
    if (threadIdx.x % 4 == 0 && r < a.M) a.lse[(size_t)blockIdx.y * a.M + r] = v;
}

// Shares from stored logits: four keys per thread
__global__ __launch_bounds__(NT) void stored_shares_kernel(ScoresArgs a)
{
    __shared__ float lse[FEW];
    const int bh = blockIdx.y, len = cache_length(a.seqlens, bh / a.HC, a.L_max), j = (blockIdx.x * NT + threadIdx.x) * 4;
    if ((int)blockIdx.x * NT * 4 >= len) return;
    const float *row = a.logits + (size_t)bh * a.M * a.pitch + min(j, ((len + 63) & ~63) - 4);
    float *out = a.scores + (size_t)bh * a.L_max + j;
    const bool wide = (a.L_max & 3) == 0 && (reinterpret_cast<uintptr_t>(a.scores) & 15) == 0 && j + 4 <= len;
    f32x4 next = *reinterpret_cast<const f32x4 *>(row), s = {0.f, 0.f, 0.f, 0.f}, old = s;
    if (wide) old = *reinterpret_cast<const f32x4 *>(out);
    merge_few(a, bh, lse);
    if (j >= len) return;
    for (int r = 0; r < a.M; ++r) {
        // (keys behind the last one that any query sees have no logits)
        const int lim = min(len, len - a.nq + r % a.nq + 1);
        const f32x4 t = next;
        if (r + 1 < a.M) next = *reinterpret_cast<const f32x4 *>(row += a.pitch);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += j + e < lim ? __builtin_amdgcn_exp2f(t[e] - lse[r]) : 0.f;
    }
    if (wide) *reinterpret_cast<f32x4 *>(out) = old + s;
    else
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (j + e < len) out[e] += s[e];
}

// Shares of 64 keys per workgroup, whose waves take every fourth tile of the queries (the next one on its way); summed in a fixed order
template <int D, typename TK, typename TQ>
__global__ __launch_bounds__(NT, (RegisterFile<D, TK, TQ, 4>::WAVES)) void shares_kernel(ScoresArgs a)
{
    __shared__ float lse[FEW];
    __shared__ float part[NW][64];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), g = lane / 16, n = lane % 16;
    int bh = blockIdx.y, at = blockIdx.x;
    by_head(bh, at);
    const int j0 = at * 64;
    const Head x = head_of(a, bh);
    if (j0 >= x.len) return;
    const bool few = a.lse == nullptr;
    if (few) merge_few(a, bh, lse);
    const char *Kh = a.K + x.b * a.sk.batch + x.h * a.sk.head;
    Operand<D, TK> k[4];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) make_operand<D, TK>(k[kt], load_words<D, TK, TK>(Kh + (int64_t)min(j0 + 16 * kt + n, x.len - 1) * a.sk.seq, g));
    const float c = tile_scale<TK>(a, bh, j0);
    f32x4 s[4];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) s[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
    // One query head: those in front of the block's first key see none of it
    const int start = a.group == 1 ? max(0, j0 - (x.len - a.nq)) / (16 * NW) * (16 * NW) : 0;
    // A lane's query, 16 NW further each time without a division
    Query r(a, start + 16 * wave + n);
    const char *row = r.row(a, x);
    const int heads = 16 * NW / a.nq, rest = 16 * NW % a.nq;
    const int64_t ahead = heads * a.sq.head + rest * a.sq.seq, wrap = a.sq.head - a.nq * a.sq.seq;
    struct Tile { Words<D, TQ> q; float ref; int lim; };
    auto load = [&](int r0) {
        Tile t;
        const int at = min(r0 + n, a.M - 1);
        t.q = load_words<D, TK, TQ>(row, g);
        t.ref = few ? lse[at & (FEW - 1)] : a.lse[(size_t)bh * a.M + at];
        t.lim = r.limit(a, x);
        r.i += rest;
        const bool over = r.i >= a.nq;
        r.i -= over ? a.nq : 0;
        r.real = r0 + 16 * NW + n < a.M;
        row += r.real ? ahead + (over ? wrap : 0) : 0;
        return t;
    };
    Tile next = load(start + 16 * wave);
    for (int r0 = start + 16 * wave; r0 < a.M; r0 += 16 * NW) {
        const Tile now = next;
        next = load(r0 + 16 * NW);
        if (__builtin_amdgcn_ballot_w64(now.lim > j0) == 0) continue;
        Operand<D, TQ> q;
        query_operand<D, TQ>(q, a, now.q);
        f32x4 t[4];
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) t[kt] = logits<D, TK, TQ>(k[kt], q);
        if (__builtin_amdgcn_ballot_w64(now.lim < j0 + 64) == 0) {
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[kt][e] += __builtin_amdgcn_exp2f(fmaf(c, t[kt][e], -now.ref));
        } else {
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(c, t[kt][e], -now.ref));
                    s[kt][e] += j0 + 16 * kt + 4 * g + e < now.lim ? p : 0.f;
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

// How a call is cut.  A wave's queries: 16 RT (fp32 queries are three operands each: two tiles of 16, otherwise four)
struct ScoresPlan {
    int M, splits, blocks;     // blocks == 0: a workgroup's waves share the queries
    bool stored;
    int64_t pitch;
    size_t stats_bytes, lse_bytes, bytes;
};

ScoresPlan scores_plan(const llla_cache &c, int H, int nq, llla_dtype in)
{
    ScoresPlan p{};
    p.M = H / c.H * nq;
    const int heads = c.B * c.H, size = c.type == LLLA_F32 ? 4 : c.type == LLLA_BF16 ? 2 : 1;
    if (p.M <= FEW) {
        // Six workgroups per compute unit, all resident (512 heads of 32768 int8 keys: 255 us; four 258, eight, in two turns, 272), of at least 1024
        // keys, or 256 while there are fewer than two per compute unit (14 heads of 4006 fp32 rows at d = 128 23 -> 13 us, 16 of 4096 int8
        // rows 8.1 -> 6.4): more parts cost their merging.
        const int wgs = std::max({1, std::min((1536 + heads - 1) / heads, (c.L_max + 1023) / 1024), std::min(512 / heads, (c.L_max + 255) / 256)});
        p.splits = NW * wgs;
        // a logit is written and read, a row of the cache would be read a second time
        p.stored = 8 * p.M <= c.d * size;
    } else {
        const int rows = 16 * (in == LLLA_F32 ? 2 : 4) * NW;
        p.blocks = (p.M + rows - 1) / rows;
        // parts of the keys, for four workgroups per compute unit (queries of a prompt see few keys or many, and two are resident: 155 us for 32 heads
        // of 4096 bf16 keys and queries; sixteen, which begin and end more often, 174, two 167), but of at least 512 keys, or 128 while there are
        // fewer workgroups than twice the compute units
        const int64_t each = (int64_t)heads * p.blocks;
        p.splits = (int)std::max<int64_t>({1, std::min<int64_t>(1024 / each, (c.L_max + 511) / 512), std::min<int64_t>(512 / each, (c.L_max + 127) / 128)});
    }
    p.pitch = p.stored ? (int64_t)(c.L_max + 63) / 64 * 64 : 0;
    p.stats_bytes = p.blocks && p.splits == 1 ? 0 : round_up((size_t)heads * p.M * 2 * p.splits * sizeof(float), 256);
    p.lse_bytes = p.blocks ? round_up((size_t)heads * p.M * sizeof(float), 256) : 0;
    p.bytes = p.stats_bytes + p.lse_bytes + round_up((size_t)heads * p.M * p.pitch * sizeof(float), 256);
    return p;
}

template <int D, typename TK, typename TQ>
hipError_t launch_scores(const ScoresProblem &p)
{
    const llla_cache &c = p.c;
    const ScoresPlan plan = scores_plan(c, p.H, p.nq, p.in);
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
    a.blocks = plan.blocks;
    a.cscale = (p.scale < 0.f ? -p.scale : p.scale) * LOG2E;
    a.negative = p.scale < 0.f ? 1 : 0;
    char *ws = static_cast<char *>(p.ws);
    a.stats = reinterpret_cast<float *>(ws);
    a.lse = plan.blocks ? reinterpret_cast<float *>(ws + plan.stats_bytes) : nullptr;
    a.logits = plan.stored ? reinterpret_cast<float *>(ws + plan.stats_bytes + plan.lse_bytes) : nullptr;
    a.pitch = plan.pitch;
    const int heads = c.B * c.H;
    if (!plan.blocks) {
        const dim3 grid(plan.splits / NW, heads);
        if (plan.M <= 16) hipLaunchKernelGGL((stats_kernel<D, TK, TQ, 1, false>), grid, dim3(NT), 0, p.stream, a);
        else if (plan.M <= 32) hipLaunchKernelGGL((stats_kernel<D, TK, TQ, 2, false>), grid, dim3(NT), 0, p.stream, a);
        else hipLaunchKernelGGL((stats_kernel<D, TK, TQ, 4, false>), grid, dim3(NT), 0, p.stream, a);
    } else {
        hipLaunchKernelGGL((stats_kernel<D, TK, TQ, RT, true>), dim3(plan.blocks * plan.splits, heads), dim3(NT), 0, p.stream, a);
        if (plan.splits > 1) hipLaunchKernelGGL(merge_stats_kernel, dim3((plan.M + NT / 4 - 1) / (NT / 4), heads), dim3(NT), 0, p.stream, a);
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

size_t cache_scores_workspace_bytes(const llla_cache &c, int H, int nq, llla_dtype in) { return scores_plan(c, H, nq, in).bytes; }

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
