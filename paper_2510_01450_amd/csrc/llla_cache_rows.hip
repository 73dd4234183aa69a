// Rows that come into a cache (llla_cache_append) and rows that stay in it (llla_cache_evict).
#include <algorithm>
#include <type_traits>

#include "llla_cache.hpp"

namespace llla {
namespace {

constexpr int NT = 256;                                   // threads of the workgroups that carry rows

template <typename C> struct IsCode { static constexpr bool value = false; };
template <> struct IsCode<Int8Code> { static constexpr bool value = true; };
template <> struct IsCode<E4m3Code> { static constexpr bool value = true; };

// A workgroup carries 64 rows of K and of V in units of sixteen features of a row: 4 D units of each tensor, K's first, dealt over the
// threads (both tensors of a row lie in whole waves at every D).
template <int D>
struct Units {
    static constexpr int ALL = 8 * D, PER_ROW = D / 16, ITER = ALL <= NT ? 1 : ALL / NT;
    static constexpr bool PARTIAL = ALL < NT;
    int tensor, row, part;
    __device__ Units(int it, int tid)
    {
        const int u = tid + NT * it;
        tensor = u / (4 * D);
        row = u % (4 * D) / PER_ROW;
        part = u % PER_ROW;
    }
};

// largest bit pattern of a wave (of absolute values: NaN above infinity above the finite ones)
__device__ __forceinline__ unsigned wave_max_bits(unsigned x)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x = max(x, (unsigned)__shfl_xor((int)x, off));
    return x;
}

__device__ __forceinline__ unsigned abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// sixteen consecutive features as numbers
template <typename TI>
__device__ __forceinline__ void load16(const TI *p, float (&x)[16])
{
    if constexpr (sizeof(TI) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 v = reinterpret_cast<const float4 *>(p)[i];
            x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint4 v = reinterpret_cast<const uint4 *>(p)[i];
            const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                x[8 * i + 2 * t] = __uint_as_float(w[t] << 16);
                x[8 * i + 2 * t + 1] = __uint_as_float(w[t] & 0xffff0000u);
            }
        }
    }
}

template <typename TC>
__device__ __forceinline__ void store16(TC *p, const float (&x)[16])
{
    if constexpr (sizeof(TC) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<float4 *>(p)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            unsigned w[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) w[t] = (unsigned)f32_to_bf16(x[8 * i + 2 * t]) | ((unsigned)f32_to_bf16(x[8 * i + 2 * t + 1]) << 16);
            reinterpret_cast<uint4 *>(p)[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

// sixteen codes of exponent `from` as codes of exponent `to`
template <typename F>
__device__ __forceinline__ uint4 shift16(uint4 w, int from, int to)
{
    unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x[4];
        decode4<F>(u[i], x);
#pragma unroll
        for (int t = 0; t < 4; ++t) x[t] = __builtin_ldexpf(x[t], from - to);
        u[i] = encode4<F>(x);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}

// ---- append ---------------------------------------------------------------------------------------------------------------------
struct AppendArgs {
    const void *k, *v;
    llla_strides sk, sv;
    void *K, *V;
    llla_strides csk, csv;
    int8_t *ke, *ve;
    float *scores;
    int32_t *pos;
    const int32_t *seqlens, *new_lens, *first_pos;
    int H, L_max, n;
};

// One workgroup per block of 64 slots that new rows may fall into: it sees all new rows of its block, so the exponent, and the codes with it, are
// written once, and no two workgroups touch a block.  Traffic is what bounds it: every value is read once and written once.
template <int D, typename TI, typename C>
__global__ __launch_bounds__(NT) void append_kernel(AppendArgs a)
{
    using U = Units<D>;
    constexpr bool CODES = IsCode<C>::value;
    const int tid = threadIdx.x, bh = blockIdx.y, b = bh / a.H, h = bh % a.H;
    const int len = a.seqlens ? min(max(a.seqlens[b], 0), a.L_max) : 0;
    const int count = a.new_lens ? min(max(a.new_lens[b], 0), a.n) : a.n;
    const int end = (int)min((int64_t)len + count, (int64_t)a.L_max);
    const int blk = len / CACHE_BLOCK + (int)blockIdx.x, base = blk * CACHE_BLOCK;
    const int s0 = max(len, base), s1 = min(end, base + CACHE_BLOCK);      // new rows of this block: slots [s0, s1)
    if (s0 >= s1) return;

    float x[U::ITER][16];
    unsigned top[2] = {0u, 0u};
#pragma unroll
    for (int it = 0; it < U::ITER; ++it) {
        const U u(it, tid);
        const int slot = base + u.row;
        const bool mine = (!U::PARTIAL || tid < U::ALL) && slot >= s0 && slot < s1;
        if (mine) {
            const llla_strides &s = u.tensor ? a.sv : a.sk;
            const TI *p = static_cast<const TI *>(u.tensor ? a.v : a.k) + b * s.batch + h * s.head + (int64_t)(slot - len) * s.seq + 16 * u.part;
            load16(p, x[it]);
            if constexpr (CODES) {
                unsigned m = 0u;
#pragma unroll
                for (int i = 0; i < 16; ++i) m = max(m, abs_bits(x[it][i]));
                if (u.tensor) top[1] = max(top[1], m);
                else top[0] = max(top[0], m);
            } else {
                const llla_strides &cs = u.tensor ? a.csv : a.csk;
                store16(static_cast<C *>(u.tensor ? a.V : a.K) + b * cs.batch + h * cs.head + (int64_t)slot * cs.seq + 16 * u.part, x[it]);
            }
        }
    }
    if constexpr (CODES) {
        __shared__ unsigned tops[2][NT / 64];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const unsigned m = wave_max_bits(top[t]);
            if (tid % 64 == 0) tops[t][tid / 64] = m;
        }
        __syncthreads();
        const bool open = len > base;                     // rows in front of the new ones share the block
        const size_t at = (size_t)bh * cache_blocks(a.L_max) + blk;
        int was[2], now[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            was[t] = open ? (int)(t ? a.ve : a.ke)[at] : EXP_LEAST;
            const unsigned m = max(max(tops[t][0], tops[t][1]), max(tops[t][2], tops[t][3]));
            now[t] = exponent_join(was[t], exponent_of<C>(__uint_as_float(m)));
        }
        __syncthreads();                                  // the old exponents are read
        if (tid < 2) (tid ? a.ve : a.ke)[at] = (int8_t)(tid ? now[1] : now[0]);
#pragma unroll
        for (int it = 0; it < U::ITER; ++it) {
            const U u(it, tid);
            if (U::PARTIAL && tid >= U::ALL) break;
            const int slot = base + u.row, e = u.tensor ? now[1] : now[0], e0 = u.tensor ? was[1] : was[0];
            const llla_strides &cs = u.tensor ? a.csv : a.csk;
            uint4 *p = reinterpret_cast<uint4 *>(static_cast<int8_t *>(u.tensor ? a.V : a.K) + b * cs.batch + h * cs.head + (int64_t)slot * cs.seq +
                                                 16 * u.part);
            if (slot >= s0 && slot < s1) {
                unsigned w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float y[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) y[t] = e == EXP_NAN ? 0.f : __builtin_ldexpf(x[it][4 * i + t], -e);
                    w[i] = encode4<C>(y);
                }
                *p = make_uint4(w[0], w[1], w[2], w[3]);
            } else if (slot < s0 && e != e0 && e != EXP_NAN) {
                *p = shift16<C>(*p, e0, e);               // (rare: a new row larger than what the block could hold)
            }
        }
    }
    if (tid < CACHE_BLOCK && base + tid >= s0 && base + tid < s1) {
        const size_t at = (size_t)bh * a.L_max + base + tid;
        if (a.scores) a.scores[at] = 0.f;
        if (a.pos) a.pos[at] = a.first_pos ? a.first_pos[b] + (base + tid - len) : base + tid;
    }
}

template <int D, typename TI, typename C>
hipError_t launch_append(const AppendProblem &p)
{
    const llla_cache &c = p.c;
    const AppendArgs a{p.k, p.v, p.sk, p.sv, c.K, c.V, c.sk, c.sv, c.k_exp, c.v_exp, c.scores, c.pos, p.seqlens, p.new_lens, p.first_pos,
                       c.H, c.L_max, p.n};
    // a sequence's new rows touch at most one block more than they fill, and no more than the cache has
    const int blocks = std::min((p.n - 1) / CACHE_BLOCK + 2, cache_blocks(c.L_max));
    hipLaunchKernelGGL((append_kernel<D, TI, C>), dim3(p.n == 1 ? 1 : blocks, c.B * c.H), dim3(NT), 0, p.stream, a);
    return hipGetLastError();
}

template <int D, typename TI>
hipError_t append_by_type(const AppendProblem &p)
{
    switch (p.c.type) {
        case LLLA_I8: return launch_append<D, TI, Int8Code>(p);
        case LLLA_E4M3: return launch_append<D, TI, E4m3Code>(p);
        case LLLA_BF16: return launch_append<D, TI, bf16_t>(p);
        default: return launch_append<D, TI, float>(p);
    }
}

template <int D>
hipError_t append_by_input(const AppendProblem &p)
{
    return p.in == LLLA_F32 ? append_by_type<D, float>(p) : append_by_type<D, bf16_t>(p);
}

// ---- evict: what stays --------------------------------------------------------------------------------------------------------------
// Workspace of one (sequence, head), in 32-bit words: header, sources, and in place also destinations and the first hole of each block
struct EvictPlan {
    int most;              // moves at most
    int blocks;            // in place: blocks of destinations
    int words;
};
constexpr int PLAN_HDR = 4;                               // moves, exponents of the block that holds slot `keep`

inline EvictPlan evict_plan(int L_max, int keep, bool in_place)
{
    EvictPlan p;
    p.most = in_place ? std::min(keep, L_max - keep) : keep;
    p.blocks = in_place ? cache_blocks(keep) : 0;
    p.words = (PLAN_HDR + p.most + (in_place ? p.most + p.blocks + 1 : 0) + 63) / 64 * 64;
    return p;
}

struct EvictArgs {
    const float *scores;
    const int32_t *pos, *seqlens;
    const int8_t *ke, *ve;             // in place, 8-bit
    int H, L_max, keep, sinks, recent, in_place;
    int32_t *lens, *index;
    EvictPlan plan;
    int *ws;
};

constexpr unsigned SAFE = 0xffffffffu;
// order-preserving, NaN below all: 0
__device__ __forceinline__ unsigned rank_of(float s)
{
    unsigned u = __float_as_uint(s);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;
    if (u == 0x80000000u) u = 0u;
    return u >> 31 ? ~u : u | 0x80000000u;
}

// The `keep` best rows of a head, and where they go.  A radix select of three digits (11, 11, 10 bits; eleven so that scores of similar size spread over
// many bins) finds the rank T of the last row that stays and how many rows of that rank do; a row's place follows from counts per
// wave of the rows that stay, or are holes (slot < keep, given up) or movers (slot >= keep, kept) in front of it.  Wave w owns a run of whole
// groups of 64 slots, so ballots count in the order of the slots, which decides between equal ranks.
// KPT > 0: the ranks of KPT groups per wave stay in registers; KPT == 0: any length, ranks are formed again in every pass.
template <int THREADS, int KPT>
__global__ __launch_bounds__(THREADS) void evict_plan_kernel(EvictArgs a)
{
    constexpr int NW = THREADS / 64, BINS = 2048, PER = BINS / THREADS;
    __shared__ unsigned hist[BINS];
    __shared__ unsigned wsum[NW];
    __shared__ int pick[2];                               // digit of T, rows of higher digits
    __shared__ int newest_s[NW];
    __shared__ int counts[NW][4];                         // rows above T and at T, each below slot keep and from there on
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int bh = blockIdx.x, b = bh / a.H;
    const int len = cache_length(a.seqlens, b, a.L_max), keep = a.keep;
    const float *scores = a.scores + (size_t)bh * a.L_max;
    const int32_t *pos = a.pos ? a.pos + (size_t)bh * a.L_max : nullptr;
    int *hdr = a.ws + (size_t)bh * a.plan.words, *src = hdr + PLAN_HDR, *dst = src + a.plan.most, *hole_of = dst + a.plan.most;
    if (bh % a.H == 0 && tid == 0) a.lens[b] = min(len, keep);
    if (a.in_place && len <= keep) {                      // nothing to give up
        if (tid == 0) hdr[0] = 0;
        for (int t = tid; t <= a.plan.blocks; t += THREADS) hole_of[t] = 0;
        if (a.index)
            for (int j = tid; j < len; j += THREADS) a.index[(size_t)bh * keep + j] = j;
        return;
    }
    const int groups = KPT > 0 ? KPT : (a.L_max + 64 * NW - 1) / (64 * NW), first = wave * groups * 64;

    int newest = len - 1;
    if (pos && a.recent > 0) {
        int m = INT32_MIN;
        for (int i = 0; i < groups; ++i) {
            const int s = first + 64 * i + lane;
            if (s < len) m = max(m, pos[s]);
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) m = max(m, __shfl_xor(m, off));
        if (lane == 0) newest_s[wave] = m;
        __syncthreads();
        newest = INT32_MIN;
#pragma unroll
        for (int w = 0; w < NW; ++w) newest = max(newest, newest_s[w]);
    }
    auto rank_at = [&](int s) {
        const int p = pos ? pos[s] : s;
        return p < a.sinks || (a.recent > 0 && (int64_t)p > (int64_t)newest - a.recent) ? SAFE : rank_of(scores[s]);
    };
    unsigned own[KPT > 0 ? KPT : 1];
    if constexpr (KPT > 0) {
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const int s = first + 64 * i + lane;
            own[i] = s < len ? rank_at(s) : 0u;
        }
    }
    auto for_groups = [&](auto fn) {                      // fn(slot, live, rank), in order
        if constexpr (KPT > 0) {
#pragma unroll
            for (int i = 0; i < KPT; ++i) {
                const int s = first + 64 * i + lane;
                fn(s, s < len, own[i]);
            }
        } else {
            for (int i = 0; i < groups; ++i) {
                const int s = first + 64 * i + lane;
                if (first + 64 * i >= len) break;
                fn(s, s < len, s < len ? rank_at(s) : 0u);
            }
        }
    };

    // the rank T of the keep-th best row; `need` of the rows of that rank stay
    const bool all = len <= keep;
    unsigned T = 0u;
    int need = keep;
    if (!all) {
#pragma unroll
        for (int digit = 0; digit < 3; ++digit) {
            const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0;
            const unsigned mask = digit == 2 ? 1023u : 2047u;
            for (int i = tid; i < BINS; i += THREADS) hist[i] = 0u;
            __syncthreads();
            for_groups([&](int, bool live, unsigned r) {
                const bool in = digit == 0 || (r >> (digit == 1 ? 21 : 10)) == (T >> (digit == 1 ? 21 : 10));
                if (live && in) atomicAdd(&hist[(r >> shift) & mask], 1u);
            });
            __syncthreads();
            // rows in the bins above this thread's, which are PER (tid ..) counted from the top
            unsigned mine = 0u, bin[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) { bin[i] = hist[BINS - 1 - (PER * tid + i)]; mine += bin[i]; }
            unsigned incl = mine;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const unsigned y = (unsigned)__shfl_up((int)incl, off);
                if (lane >= off) incl += y;
            }
            if (lane == 63) wsum[wave] = incl;
            __syncthreads();
            unsigned above = incl - mine;
#pragma unroll
            for (int w = 0; w < NW; ++w) above += w < wave ? wsum[w] : 0u;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (above < (unsigned)need && above + bin[i] >= (unsigned)need) {      // one bin of one thread
                    pick[0] = BINS - 1 - (PER * tid + i);
                    pick[1] = (int)above;
                }
                above += bin[i];
            }
            __syncthreads();
            T |= (unsigned)pick[0] << shift;
            need -= pick[1];
        }
    }

    // rows per wave, below slot keep and from there on
    {
        int gl = 0, gh = 0, el = 0, eh = 0;
        for_groups([&](int s, bool live, unsigned r) {
            const bool gt = live && (all || r > T), eq = live && !all && r == T;
            gl += __builtin_popcountll(__builtin_amdgcn_ballot_w64(gt && s < keep));
            gh += __builtin_popcountll(__builtin_amdgcn_ballot_w64(gt && s >= keep));
            el += __builtin_popcountll(__builtin_amdgcn_ballot_w64(eq && s < keep));
            eh += __builtin_popcountll(__builtin_amdgcn_ballot_w64(eq && s >= keep));
        });
        if (lane == 0) { counts[wave][0] = gl; counts[wave][1] = gh; counts[wave][2] = el; counts[wave][3] = eh; }
    }
    __syncthreads();
    int equal = 0, kept = 0, kept_high = 0, kept_low = 0; // in front of this wave: rows of rank T; rows that stay, also by side
    {
        int e = 0;
        for (int w = 0; w < NW; ++w) {
            const int el = counts[w][2], eh = counts[w][3];
            const int tl = min(max(need - e, 0), el), th = min(max(need - e - el, 0), eh);
            if (w < wave) {
                equal += el + eh;
                kept_low += counts[w][0] + tl;
                kept_high += counts[w][1] + th;
            }
            e += el + eh;
        }
        kept = kept_low + kept_high;
    }
    int holes = min(min(first, keep), len) - kept_low, movers = kept_high;
    const uint64_t below = (1ull << lane) - 1;
    for_groups([&](int s, bool live, unsigned r) {
        const bool eq = live && !all && r == T;
        const uint64_t me = __builtin_amdgcn_ballot_w64(eq);
        const bool stays = live && (all || r > T || (eq && equal + __builtin_popcountll(me & below) < need));
        equal += __builtin_popcountll(me);
        if (!a.in_place) {
            const uint64_t m = __builtin_amdgcn_ballot_w64(stays);
            if (stays) {
                const int j = kept + __builtin_popcountll(m & below);
                src[j] = s;
                if (a.index) a.index[(size_t)bh * keep + j] = s;
            }
            kept += __builtin_popcountll(m);
        } else {
            const bool hole = live && !stays && s < keep, mover = stays && s >= keep;
            const uint64_t mh = __builtin_amdgcn_ballot_w64(hole), mm = __builtin_amdgcn_ballot_w64(mover);
            if (lane == 0 && s / 64 < a.plan.blocks) hole_of[s / 64] = holes;
            if (hole) dst[holes + __builtin_popcountll(mh & below)] = s;
            if (mover) src[movers + __builtin_popcountll(mm & below)] = s;
            if (a.index && stays && s < keep) a.index[(size_t)bh * keep + s] = s;
            holes += __builtin_popcountll(mh);
            movers += __builtin_popcountll(mm);
        }
    });
    if (wave == NW - 1 && lane == 0) {                    // (the last wave's counts end with all rows)
        hdr[0] = a.in_place ? movers : kept;
        if (a.in_place) {
            hole_of[a.plan.blocks] = holes;
            if (a.ke) {
                const size_t at = (size_t)bh * cache_blocks(a.L_max) + keep / CACHE_BLOCK;      // (len > keep: the slot exists)
                hdr[1] = a.ke[at];
                hdr[2] = a.ve[at];
            }
        }
    }
}

// ---- evict: rows that move ----------------------------------------------------------------------------------------------------------
struct MoveArgs {
    const void *K, *V;
    void *Kd, *Vd;
    llla_strides sk, sv, dk, dv;
    const int8_t *ke, *ve;
    int8_t *ked, *ved;
    const float *scores;
    const int32_t *pos;
    float *scores_d;
    int32_t *pos_d, *index;            // index: in place only (the plan writes it otherwise)
    int H, L_max, Ld_max, keep, in_place;
    EvictPlan plan;
    const int *ws;
};

__device__ __forceinline__ void move_row_words(const MoveArgs &a, int bh, int from, int to)
{
    const size_t f = (size_t)bh * a.L_max + from, t = (size_t)bh * a.Ld_max + to;
    if (a.scores_d) a.scores_d[t] = a.scores[f];
    if (a.pos_d) a.pos_d[t] = a.pos ? a.pos[f] : from;
    if (a.index) a.index[(size_t)bh * a.keep + to] = from;
}

// Rows of numbers: copies, MOVE_ROWS of a head per workgroup, sixteen bytes per thread at a time
constexpr int MOVE_ROWS = 32;
template <int ROW_BYTES>
__global__ __launch_bounds__(NT) void move_kernel(MoveArgs a)
{
    constexpr int PER_ROW = ROW_BYTES / 16, ALL = 2 * MOVE_ROWS * PER_ROW, ITER = (ALL + NT - 1) / NT;
    const int tid = threadIdx.x, bh = blockIdx.y, b = bh / a.H, h = bh % a.H, i0 = blockIdx.x * MOVE_ROWS;
    const int *hdr = a.ws + (size_t)bh * a.plan.words, *src = hdr + PLAN_HDR, *dst = src + a.plan.most;
    const int count = min(hdr[0] - i0, MOVE_ROWS);
    if (count <= 0) return;
    uint4 v[ITER];
    char *to[ITER];
#pragma unroll
    for (int it = 0; it < ITER; ++it) {
        const int u = tid + NT * it, tensor = u / (MOVE_ROWS * PER_ROW), r = u % (MOVE_ROWS * PER_ROW) / PER_ROW, part = u % PER_ROW;
        to[it] = nullptr;
        if (u < ALL && r < count) {
            const int s = src[i0 + r], d = a.in_place ? dst[i0 + r] : i0 + r;
            const llla_strides &ss = tensor ? a.sv : a.sk, &ds = tensor ? a.dv : a.dk;      // (in bytes)
            v[it] = *reinterpret_cast<const uint4 *>(static_cast<const char *>(tensor ? a.V : a.K) + b * ss.batch + h * ss.head + (int64_t)s * ss.seq + 16 * part);
            to[it] = static_cast<char *>(tensor ? a.Vd : a.Kd) + b * ds.batch + h * ds.head + (int64_t)d * ds.seq + 16 * part;
        }
    }
#pragma unroll
    for (int it = 0; it < ITER; ++it)
        if (to[it]) *reinterpret_cast<uint4 *>(to[it]) = v[it];
    if (tid < count) move_row_words(a, bh, src[i0 + tid], a.in_place ? dst[i0 + tid] : i0 + tid);
}

// Rows of codes: one workgroup per block of destinations.  A row needs the exponent that its own largest code asks for, not its old block's, so a
// block's exponent only grows for rows that do not fit it.
template <int D, typename F>
__global__ __launch_bounds__(NT) void move_codes_kernel(MoveArgs a)
{
    using U = Units<D>;
    __shared__ int from_s[CACHE_BLOCK];
    __shared__ int needs[2][NT / 64];
    const int tid = threadIdx.x, bh = blockIdx.y, b = bh / a.H, h = bh % a.H, blk = blockIdx.x, base = blk * CACHE_BLOCK;
    const int *hdr = a.ws + (size_t)bh * a.plan.words, *src = hdr + PLAN_HDR, *dst = src + a.plan.most, *hole_of = dst + a.plan.most;
    int i0 = base, count;
    if (a.in_place) {
        i0 = hole_of[blk];
        count = hole_of[blk + 1] - i0;
    } else {
        count = min(hdr[0] - base, CACHE_BLOCK);
    }
    if (count <= 0) return;
    if (tid < CACHE_BLOCK) from_s[tid] = -1;
    __syncthreads();
    if (tid < count) {
        const int s = src[i0 + tid], d = a.in_place ? dst[i0 + tid] : i0 + tid;
        from_s[d - base] = s;
        move_row_words(a, bh, s, d);
    }
    __syncthreads();
    const size_t exps = (size_t)bh * cache_blocks(a.L_max);
    uint4 w[U::ITER];
    int from[U::ITER], e0[U::ITER];
    int need[2] = {EXP_LEAST, EXP_LEAST};
#pragma unroll
    for (int it = 0; it < U::ITER; ++it) {
        const U u(it, tid);
        from[it] = -1;
        if (!U::PARTIAL || tid < U::ALL) from[it] = from_s[u.row];
        unsigned m = 0u;
        e0[it] = EXP_LEAST;
        if (from[it] >= 0) {
            const llla_strides &ss = u.tensor ? a.sv : a.sk;
            w[it] = *reinterpret_cast<const uint4 *>(static_cast<const int8_t *>(u.tensor ? a.V : a.K) + b * ss.batch + h * ss.head +
                                                     (int64_t)from[it] * ss.seq + 16 * u.part);
            // (in place the block of slot keep may be getting another exponent in these moments: as the plan saw it)
            const int fb = from[it] / CACHE_BLOCK;
            e0[it] = a.in_place && fb == a.keep / CACHE_BLOCK ? hdr[1 + u.tensor] : (int)(u.tensor ? a.ve : a.ke)[exps + fb];
            const unsigned v[4] = {w[it].x, w[it].y, w[it].z, w[it].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x[4];
                decode4<F>(v[i], x);
#pragma unroll
                for (int t = 0; t < 4; ++t) m = max(m, abs_bits(x[t]));
            }
        }
        // of these sixteen codes; the block takes the largest anyway
        int n = m == 0u ? EXP_LEAST : exponent_of<F>(__uint_as_float(m));
        if (e0[it] == EXP_NAN) n = EXP_NAN;
        else if (n != EXP_NAN && m != 0u) n = max(n + e0[it], EXP_LEAST);
        need[0] = u.tensor ? need[0] : exponent_join(need[0], n);
        need[1] = u.tensor ? exponent_join(need[1], n) : need[1];
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) need[t] = exponent_join(need[t], __shfl_xor(need[t], off));
        if (tid % 64 == 0) needs[t][tid / 64] = need[t];
    }
    const size_t at = (size_t)bh * cache_blocks(a.Ld_max) + blk;
    int was[2] = {EXP_LEAST, EXP_LEAST};
    if (a.in_place) { was[0] = a.ked[at]; was[1] = a.ved[at]; }
    __syncthreads();                                      // (and the old exponents are read)
    int now[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
        now[t] = exponent_join(was[t], exponent_join(exponent_join(needs[t][0], needs[t][1]), exponent_join(needs[t][2], needs[t][3])));
    if (tid < 2) (tid ? a.ved : a.ked)[at] = (int8_t)(tid ? now[1] : now[0]);
#pragma unroll
    for (int it = 0; it < U::ITER; ++it) {
        const U u(it, tid);
        if (U::PARTIAL && tid >= U::ALL) break;
        const int slot = base + u.row, e = u.tensor ? now[1] : now[0], eb = u.tensor ? was[1] : was[0];
        const llla_strides &ds = u.tensor ? a.dv : a.dk;
        uint4 *p = reinterpret_cast<uint4 *>(static_cast<int8_t *>(u.tensor ? a.Vd : a.Kd) + b * ds.batch + h * ds.head + (int64_t)slot * ds.seq + 16 * u.part);
        if (from[it] >= 0) *p = e == EXP_NAN || e == e0[it] ? w[it] : shift16<F>(w[it], e0[it], e);
        else if (a.in_place && slot < a.keep && e != eb && e != EXP_NAN) *p = shift16<F>(*p, eb, e);
    }
}

template <int D>
hipError_t launch_moves(const EvictProblem &p, MoveArgs a)
{
    const int bh = p.c.B * p.c.H, size = p.c.type == LLLA_F32 ? 4 : p.c.type == LLLA_BF16 ? 2 : 1;
    if (size == 1) {
        const dim3 grid(cache_blocks(p.keep), bh);
        if (p.c.type == LLLA_I8) hipLaunchKernelGGL((move_codes_kernel<D, Int8Code>), grid, dim3(NT), 0, p.stream, a);
        else hipLaunchKernelGGL((move_codes_kernel<D, E4m3Code>), grid, dim3(NT), 0, p.stream, a);
    } else {
        for (llla_strides *s : {&a.sk, &a.sv, &a.dk, &a.dv}) { s->batch *= size; s->head *= size; s->seq *= size; }
        const dim3 grid((a.plan.most + MOVE_ROWS - 1) / MOVE_ROWS, bh);
        if (size == 2) hipLaunchKernelGGL((move_kernel<2 * D>), grid, dim3(NT), 0, p.stream, a);
        else hipLaunchKernelGGL((move_kernel<4 * D>), grid, dim3(NT), 0, p.stream, a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t cache_append(const AppendProblem &p)
{
    switch (p.c.d) {
        case 16: return append_by_input<16>(p);
        case 32: return append_by_input<32>(p);
        case 64: return append_by_input<64>(p);
        case 128: return append_by_input<128>(p);
        default: return hipErrorInvalidValue;
    }
}

size_t cache_evict_workspace_bytes(const llla_cache &c, int keep)
{
    // of the two forms the one that needs more
    const int words = std::max(evict_plan(c.L_max, keep, true).words, evict_plan(c.L_max, keep, false).words);
    return round_up((size_t)c.B * c.H * words * sizeof(int), 256);
}

hipError_t cache_evict(const EvictProblem &p)
{
    const llla_cache &c = p.c, &d = p.in_place ? p.c : p.into;
    const bool codes = c.type == LLLA_I8 || c.type == LLLA_E4M3;
    const EvictPlan plan = evict_plan(c.L_max, p.keep, p.in_place);
    const int bh = c.B * c.H;
    const EvictArgs a{c.scores, c.pos, p.seqlens, codes && p.in_place ? c.k_exp : nullptr, codes && p.in_place ? c.v_exp : nullptr, c.H, c.L_max,
                      p.keep, p.sinks, p.recent, p.in_place ? 1 : 0, p.lens, p.index, plan, static_cast<int *>(p.ws)};
    const dim3 grid(bh);
    if (c.L_max <= 1024) hipLaunchKernelGGL((evict_plan_kernel<256, 4>), grid, dim3(256), 0, p.stream, a);
    else if (c.L_max <= 4096) hipLaunchKernelGGL((evict_plan_kernel<256, 16>), grid, dim3(256), 0, p.stream, a);
    else if (c.L_max <= 16384) hipLaunchKernelGGL((evict_plan_kernel<1024, 16>), grid, dim3(1024), 0, p.stream, a);
    else hipLaunchKernelGGL((evict_plan_kernel<1024, 0>), grid, dim3(1024), 0, p.stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || plan.most == 0) return e;
    const MoveArgs m{c.K, c.V, d.K, d.V, c.sk, c.sv, d.sk, d.sv, c.k_exp, c.v_exp, d.k_exp, d.v_exp, c.scores, c.pos, d.scores, d.pos,
                     p.in_place ? p.index : nullptr, c.H, c.L_max, d.L_max, p.keep, p.in_place ? 1 : 0, plan, static_cast<const int *>(p.ws)};
    switch (c.d) {
        case 16: return launch_moves<16>(p, m);
        case 32: return launch_moves<32>(p, m);
        case 64: return launch_moves<64>(p, m);
        case 128: return launch_moves<128>(p, m);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace llla
