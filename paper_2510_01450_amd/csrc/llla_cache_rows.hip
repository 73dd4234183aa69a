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
// written once, and no two workgroups touch a block.  Traffic is what bounds it: every value is read once and written once (128 heads x 1535 bf16 rows
// of 64 to int8 17 us, 4.4 TB/s read and written; one token of 512 heads 5 us, its launch).
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
// Workspace of one (sequence, head), in 32-bit words: header, sources, and in place also destinations and the first hole of each block;
// for long caches also what the launches of the selection hand on
struct EvictPlan {
    int most;              // moves at most
    int blocks;            // in place: blocks of destinations
    int chunks;            // workgroups of a head, 0: one for the head
    int state;             // offset of the state of the selection
    int words;
};
constexpr int PLAN_HDR = 4;                               // moves, exponents of the block that holds slot `keep`
constexpr int BINS = 2048, HISTS = 3 * BINS, CHOICES = 4 * 5;      // histograms, and the choice of each step

constexpr int CHUNK = 2048;                               // slots of a workgroup where a head has several
// One workgroup holds the ranks of up to 16384 slots in registers and selects in one launch; longer rows take six launches of a workgroup per
// CHUNK.  us, one launch / six: 64 heads x 16384 slots 23 / 35, 512 heads 44 / 117; 64 heads x 32768, where 32 ranks a thread no longer fit, 112 / 43.
constexpr int ONE_LAUNCH = 16384;

inline EvictPlan evict_plan(int L_max, int keep, bool in_place)
{
    EvictPlan p;
    p.most = in_place ? std::min(keep, L_max - keep) : keep;
    p.blocks = in_place ? cache_blocks(keep) : 0;
    p.chunks = L_max <= ONE_LAUNCH ? 0 : (L_max + CHUNK - 1) / CHUNK;
    p.state = PLAN_HDR + p.most + (in_place ? p.most + p.blocks + 1 : 0);
    p.words = (p.state + (p.chunks ? HISTS + CHOICES + 5 * p.chunks : 0) + 63) / 64 * 64;
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

__device__ __forceinline__ int wave_max_int(int x)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x = max(x, __shfl_xor(x, off));
    return x;
}

__device__ __forceinline__ int popcount64(uint64_t m) { return __builtin_popcountll(m); }

// One head as a workgroup sees it
struct EvictHead {
    int bh, len;
    const float *scores;
    const int32_t *pos;
    int *hdr, *src, *dst, *hole_of, *state;
    __device__ EvictHead(const EvictArgs &a, int bh_) : bh(bh_)
    {
        len = cache_length(a.seqlens, bh / a.H, a.L_max);
        scores = a.scores + (size_t)bh * a.L_max;
        pos = a.pos ? a.pos + (size_t)bh * a.L_max : nullptr;
        hdr = a.ws + (size_t)bh * a.plan.words;
        src = hdr + PLAN_HDR;
        dst = src + a.plan.most;
        hole_of = dst + a.plan.most;
        state = hdr + a.plan.state;
    }
};

// Positions and scores of KPT groups of 64 slots, as ranks.  (Every load has a valid address and no condition around it, so that all are in flight
// together: with a condition each was waited for, 16 trips to memory one after the other, 34 us for 256 heads of 4160 rows.)
template <int KPT>
struct Ranks {
    unsigned own[KPT];
    int p[KPT];
    __device__ void load(const EvictHead &x, int first, int lane)
    {
        const int last = x.len - 1;
#pragma unroll
        for (int i = 0; i < KPT; ++i) own[i] = __float_as_uint(x.scores[min(first + 64 * i + lane, last)]);
#pragma unroll
        for (int i = 0; i < KPT; ++i) p[i] = x.pos ? x.pos[min(first + 64 * i + lane, last)] : first + 64 * i + lane;
    }
    __device__ int newest(const EvictHead &x, int first, int lane) const
    {
        int m = INT32_MIN;
#pragma unroll
        for (int i = 0; i < KPT; ++i) m = first + 64 * i + lane < x.len ? max(m, p[i]) : m;
        return wave_max_int(m);
    }
    __device__ void rank(const EvictArgs &a, int newest)
    {
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const bool safe = p[i] < a.sinks || (a.recent > 0 && (int64_t)p[i] > (int64_t)newest - a.recent);
            own[i] = safe ? SAFE : rank_of(__uint_as_float(own[i]));
        }
    }
};

// Digits of a rank: 11, 11 and 10 bits; eleven so that scores of similar size spread over many bins
__device__ __forceinline__ int digit_shift(int digit) { return digit == 0 ? 21 : digit == 1 ? 10 : 0; }
__device__ __forceinline__ unsigned digit_mask(int digit) { return digit == 2 ? 1023u : 2047u; }

// What is known of the rank T of the last row that stays: rows above T stay, and the first `need` of rank T
struct Choice {
    unsigned T;
    int need;
    bool done;             // T is final
};

// Narrows the choice by the histogram of the digit, of which a thread has its own PER bins, counted from the top.  All threads of the workgroup;
// pick, wsum: LDS.
template <int THREADS>
struct Bins {
    static constexpr int PER = BINS / THREADS;
    unsigned v[PER];
    __device__ void load(const unsigned *hist)
    {
#pragma unroll
        for (int i = 0; i < PER; ++i) v[i] = hist[BINS - 1 - (PER * (int)threadIdx.x + i)];
    }
};
template <int THREADS>
__device__ __forceinline__ void narrow(Choice &c, int digit, const Bins<THREADS> &b, unsigned *wsum, int *pick)
{
    constexpr int NW = THREADS / 64, PER = Bins<THREADS>::PER;
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    const auto &bin = b.v;
    unsigned mine = 0u;
#pragma unroll
    for (int i = 0; i < PER; ++i) mine += bin[i];
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
        if (above < (unsigned)c.need && above + bin[i] >= (unsigned)c.need) {      // one bin of one thread
            pick[0] = BINS - 1 - (PER * tid + i);
            pick[1] = (int)above;
            pick[2] = (int)bin[i];
        }
        above += bin[i];
    }
    __syncthreads();
    c.T |= (unsigned)pick[0] << digit_shift(digit);
    c.need -= pick[1];
    if (digit < 2 && pick[2] == c.need && c.T > 0u) {      // all rows of the bin stay: those above the rank in front of it (one of zero never does)
        c.T -= 1u;
        c.need = 0;
        c.done = true;
    }
    __syncthreads();                                      // (pick is free again)
}

template <int KPT>
__device__ __forceinline__ void count_digit(const Ranks<KPT> &r, const EvictHead &x, int first, int lane, int digit, const Choice &c, unsigned *hist)
{
    const int shift = digit_shift(digit), before = digit == 1 ? 21 : 10;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        const bool in = first + 64 * i + lane < x.len && (digit == 0 || r.own[i] >> before == c.T >> before);
        if (in) atomicAdd(&hist[(r.own[i] >> shift) & digit_mask(digit)], 1u);
    }
}

// A group of 64 slots as bit masks: rows above T, rows at T, slots below `keep`.  Scalar, like all that is counted from them.
struct Group { uint64_t gt, eq, low; };
template <int KPT>
__device__ __forceinline__ Group group_of(const Ranks<KPT> &r, const EvictHead &x, int i, int first, int lane, int keep, bool all, const Choice &c)
{
    const int s0 = first + 64 * i;
    auto bits = [](int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; };
    const uint64_t live = bits(x.len - s0);
    if (all) return Group{live, 0ull, bits(keep - s0)};
    return Group{live & __builtin_amdgcn_ballot_w64(r.own[i] > c.T), live & __builtin_amdgcn_ballot_w64(r.own[i] == c.T), bits(keep - s0)};
}

// rows above T and at T, each below slot keep and from there on
struct Counts { int gl, gh, el, eh; };
template <int KPT>
__device__ __forceinline__ Counts count_sides(const Ranks<KPT> &r, const EvictHead &x, int first, int lane, int keep, bool all, const Choice &c)
{
    Counts n{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        if (first + 64 * i < x.len) {                     // (a scalar branch)
            const Group g = group_of(r, x, i, first, lane, keep, all, c);
            n.gl += popcount64(g.gt & g.low);
            n.gh += popcount64(g.gt & ~g.low);
            n.el += popcount64(g.eq & g.low);
            n.eh += popcount64(g.eq & ~g.low);
        }
    }
    return n;
}

// Rows in front of a run of slots: of rank T; that stay, by side of slot keep
struct Front { int equal, low, high; };
__device__ __forceinline__ void advance(Front &f, const Counts &n, int need)
{
    const int tl = min(max(need - f.equal, 0), n.el), th = min(max(need - f.equal - n.el, 0), n.eh);
    f.equal += n.el + n.eh;
    f.low += n.gl + tl;
    f.high += n.gh + th;
}

// number of a mask's bits below the lane
__device__ __forceinline__ int bits_below(uint64_t m)
{
    return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0u));
}

// A row's place follows from the rows in front of it that stay, or are holes (slot < keep, given up) or movers (slot >= keep, kept)
template <int KPT>
__device__ __forceinline__ void place(const EvictArgs &a, const EvictHead &x, const Ranks<KPT> &r, int first, int lane, bool all, const Choice &c, Front f,
                                      bool last)
{
    const int keep = a.keep;
    int kept = f.low + f.high, holes = min(min(first, keep), x.len) - f.low, movers = f.high, equal = f.equal;
    auto mine = [&](uint64_t m) { return ((m >> lane) & 1) != 0; };
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        const int s0 = first + 64 * i, s = s0 + lane;
        if (s0 < x.len) {                                 // (scalar branches)
            const Group g = group_of(r, x, i, first, lane, keep, all, c);
            uint64_t stay = g.gt;
            if (g.eq != 0) {
                if (equal < c.need) stay |= g.eq & __builtin_amdgcn_ballot_w64(equal + bits_below(g.eq) < c.need);
                equal += popcount64(g.eq);
            }
            if (!a.in_place) {
                if (mine(stay)) {
                    const int j = kept + bits_below(stay);
                    x.src[j] = s;
                    if (a.index) a.index[(size_t)x.bh * keep + j] = s;
                }
                kept += popcount64(stay);
            } else {
                const uint64_t hole = ~stay & g.low, mover = stay & ~g.low;      // (more rows than keep: the slots below it are all taken)
                if (lane == 0 && s0 / 64 < a.plan.blocks) x.hole_of[s0 / 64] = holes;
                if (mine(hole)) x.dst[holes + bits_below(hole)] = s;
                if (mine(mover)) x.src[movers + bits_below(mover)] = s;
                if (a.index && mine(stay & g.low)) a.index[(size_t)x.bh * keep + s] = s;
                holes += popcount64(hole);
                movers += popcount64(mover);
            }
        }
    }
    if (last && lane == 0) {                              // (the last run's counts end with all rows)
        x.hdr[0] = a.in_place ? movers : kept;
        if (a.in_place) {
            x.hole_of[a.plan.blocks] = holes;
            if (a.ke) {
                const size_t at = (size_t)x.bh * cache_blocks(a.L_max) + keep / CACHE_BLOCK;      // (more rows than keep: the slot exists)
                x.hdr[1] = a.ke[at];
                x.hdr[2] = a.ve[at];
            }
        }
    }
}

// Lengths, and heads that have nothing to select; true: done
template <int THREADS>
__device__ __forceinline__ bool evict_early(const EvictArgs &a, const EvictHead &x)
{
    const int tid = threadIdx.x;
    if (x.bh % a.H == 0 && tid == 0) a.lens[x.bh / a.H] = min(x.len, a.keep);
    if (x.len == 0 || (a.in_place && x.len <= a.keep)) {
        if (tid == 0) x.hdr[0] = 0;
        for (int t = tid; a.in_place && t <= a.plan.blocks; t += THREADS) x.hole_of[t] = 0;
        if (a.index)
            for (int j = tid; j < x.len; j += THREADS) a.index[(size_t)x.bh * a.keep + j] = j;
        return true;
    }
    return false;
}

// The `keep` best rows of a head, and where they go: a radix select finds the rank of the last row that stays, then every row's place follows from
// counts per wave.  Wave w owns a run of whole groups of 64 slots, so ballots count in the order of the slots, which decides between equal ranks.
template <int THREADS, int KPT>
__global__ __launch_bounds__(THREADS) void evict_plan_kernel(EvictArgs a)
{
    constexpr int NW = THREADS / 64;
    __shared__ unsigned hist[BINS];
    __shared__ unsigned wsum[NW];
    __shared__ int pick[3];
    __shared__ int newest_s[NW];
    __shared__ Counts counts[NW];
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const EvictHead x(a, blockIdx.x);
    if (evict_early<THREADS>(a, x)) return;
    const int first = wave * KPT * 64;
    Ranks<KPT> r;
    r.load(x, first, lane);
    int newest = x.len - 1;
    if (x.pos && a.recent > 0) {
        const int m = r.newest(x, first, lane);
        if (lane == 0) newest_s[wave] = m;
        __syncthreads();
        newest = INT32_MIN;
#pragma unroll
        for (int w = 0; w < NW; ++w) newest = max(newest, newest_s[w]);
    }
    r.rank(a, newest);
    const bool all = x.len <= a.keep;
    Choice c{0u, a.keep, all};
#pragma unroll 1
    for (int digit = 0; digit < 3 && !c.done; ++digit) {
        for (int i = tid; i < BINS; i += THREADS) hist[i] = 0u;
        __syncthreads();
        count_digit(r, x, first, lane, digit, c, hist);
        __syncthreads();
        Bins<THREADS> bins;
        bins.load(hist);
        narrow<THREADS>(c, digit, bins, wsum, pick);
    }
    const Counts n = count_sides(r, x, first, lane, a.keep, all, c);
    if (lane == 0) counts[wave] = n;
    __syncthreads();
    Front f{0, 0, 0};
    for (int w = 0; w < wave; ++w) advance(f, counts[w], c.need);
    place(a, x, r, first, lane, all, c, f, wave == NW - 1);
}

// The same for long caches, a head dealt over workgroups of CHUNK slots, in six launches: step 0 newest positions (and histograms cleared), 1 to 3 the
// digits, 4 counts, 5 places.  Every workgroup reads the histogram of the step before and narrows the choice for itself.
// state: histograms, choice of each step, newest position of each chunk, counts of each chunk
__global__ __launch_bounds__(NT) void evict_long_kernel(EvictArgs a, int step)
{
    constexpr int KPT = CHUNK / NT, NWG = NT / 64;
    __shared__ unsigned hist[BINS];
    __shared__ unsigned wsum[NWG];
    __shared__ int pick[3];
    __shared__ Counts counts[NWG];
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64), chunk = blockIdx.x;
    const EvictHead x(a, blockIdx.y);
    int *choice_of = x.state + HISTS, *newest_of = choice_of + CHOICES;
    Counts *counts_of = reinterpret_cast<Counts *>(newest_of + a.plan.chunks);
    unsigned *hists = reinterpret_cast<unsigned *>(x.state);
    if (step == 0) {
        for (int i = chunk * NT + tid; i < HISTS; i += a.plan.chunks * NT) hists[i] = 0u;
        if (chunk == 0) evict_early<NT>(a, x);
    }
    if (x.len == 0 || (a.in_place && x.len <= a.keep)) return;
    const int first = chunk * CHUNK + wave * KPT * 64;
    const bool all = x.len <= a.keep, live = chunk * CHUNK < x.len;
    Ranks<KPT> r;
    if (step == 0) {
        if (!x.pos || a.recent == 0) return;
        r.load(x, first, lane);
        const int m = r.newest(x, first, lane);
        if (lane == 0) wsum[wave] = (unsigned)m;
        __syncthreads();
        if (tid == 0) newest_of[chunk] = max(max((int)wsum[0], (int)wsum[1]), max((int)wsum[2], (int)wsum[3]));
        return;
    }
    if (!live && step < 3) return;
    // what the step reads, all requested together: a trip to memory is a fifth of it
    r.load(x, first, lane);
    Bins<NT> bins;
    bins.load(hists + (step < 2 ? 0 : min(step - 2, 2)) * BINS);
    const bool by_age = x.pos && a.recent > 0;
    int newest = INT32_MIN;
    if (by_age) newest = newest_of[min(lane, a.plan.chunks - 1)];
    const int *before = choice_of + 4 * (step - 1);
    const Choice told{(unsigned)before[0], before[1], before[2] != 0};
    const bool placed = choice_of[4 * 3 + 2] != 0;
    // The choice that the step before began with, narrowed by what it counted.  Ordinarily two digits tell (scores differ): step 3 then counts the rows that
    // stay, step 4 gives them their places, and the last step has nothing left to do.
    if (step == 5 && placed) return;
    Choice c = step <= 2 ? Choice{0u, a.keep, all} : told;
    const bool counted = step == 5 || (step == 4 && c.done);
    if (step >= 2 && step <= 4) {
        if (!c.done) {
            narrow<NT>(c, step - 2, bins, wsum, pick);
        }
        if (chunk == 0 && tid == 0) {
            choice_of[4 * step] = (int)c.T;
            choice_of[4 * step + 1] = c.need;
            choice_of[4 * step + 2] = c.done ? 1 : 0;
        }
    }
    for (int i = lane + 64; by_age && i < a.plan.chunks; i += 64) newest = max(newest, newest_of[i]);
    r.rank(a, by_age ? wave_max_int(newest) : x.len - 1);
    if (step <= 2 || (step == 3 && !c.done)) {
        if (c.done || !live) return;
        for (int i = tid; i < BINS; i += NT) hist[i] = 0u;
        __syncthreads();
        count_digit(r, x, first, lane, step - 1, c, hist);
        __syncthreads();
        for (int i = tid; i < BINS; i += NT)
            if (hist[i]) atomicAdd(&hists[(step - 1) * BINS + i], hist[i]);
        return;
    }
    const Counts n = count_sides(r, x, first, lane, a.keep, all, c);
    if (lane == 0) counts[wave] = n;
    __syncthreads();
    if (!counted) {
        if (tid == 0) {
            Counts s = counts[0];
            for (int w = 1; w < NWG; ++w) { s.gl += counts[w].gl; s.gh += counts[w].gh; s.el += counts[w].el; s.eh += counts[w].eh; }
            counts_of[chunk] = s;
        }
        return;
    }
    // what is in front of the chunk: sums of the chunks, those of rank T that stay as one run below slot keep and one from there on
    Front f{0, 0, 0};
    {
        int gl = 0, gh = 0, el = 0, eh = 0;
        for (int i = lane; i < chunk; i += 64) {
            const Counts k = counts_of[i];
            gl += k.gl; gh += k.gh; el += k.el; eh += k.eh;
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            gl += __shfl_xor(gl, off); gh += __shfl_xor(gh, off); el += __shfl_xor(el, off); eh += __shfl_xor(eh, off);
        }
        advance(f, Counts{gl, gh, el, eh}, c.need);
    }
    for (int w = 0; w < wave; ++w) advance(f, counts[w], c.need);
    place(a, x, r, first, lane, all, c, f, chunk == a.plan.chunks - 1 && wave == NWG - 1);
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

// Rows of numbers: copies, MOVE_ROWS of a head per workgroup, sixteen bytes per thread at a time (64 heads x 4096 rows of 256 bytes, keys and values:
// 63 us, 4.3 TB/s read and written)
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

// Exponent that sixteen codes of exponent e ask for (EXP_LEAST for zeros).  A row needs the exponent that its own largest code asks for, not its
// old block's, so a block's exponent only grows for rows that do not fit it.
template <typename F>
__device__ __forceinline__ int exponent_needed(uint4 w, int e)
{
    const unsigned v[4] = {w.x, w.y, w.z, w.w};
    unsigned m = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x[4];
        decode4<F>(v[i], x);
#pragma unroll
        for (int t = 0; t < 4; ++t) m = max(m, abs_bits(x[t]));
    }
    if (e == EXP_NAN) return EXP_NAN;
    if (m == 0u) return EXP_LEAST;
    const int n = exponent_of<F>(__uint_as_float(m));
    return n == EXP_NAN ? EXP_NAN : max(n + e, EXP_LEAST);
}

__device__ __forceinline__ int wave_join(int e)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) e = exponent_join(e, __shfl_xor(e, off));
    return e;
}

// Rows of codes into another cache: one workgroup per block of destinations
template <int D, typename F>
__global__ __launch_bounds__(NT) void move_codes_kernel(MoveArgs a)
{
    using U = Units<D>;
    __shared__ int needs[2][NT / 64];
    const int tid = threadIdx.x, bh = blockIdx.y, b = bh / a.H, h = bh % a.H, blk = blockIdx.x, base = blk * CACHE_BLOCK;
    const int *hdr = a.ws + (size_t)bh * a.plan.words, *src = hdr + PLAN_HDR;
    const int count = min(hdr[0] - base, CACHE_BLOCK);
    if (count <= 0) return;
    if (tid < count) move_row_words(a, bh, src[base + tid], base + tid);
    const size_t exps = (size_t)bh * cache_blocks(a.L_max);
    uint4 w[U::ITER];
    int e0[U::ITER];
    int need[2] = {EXP_LEAST, EXP_LEAST};
#pragma unroll
    for (int it = 0; it < U::ITER; ++it) {
        const U u(it, tid);
        const bool mine = (!U::PARTIAL || tid < U::ALL) && u.row < count;
        const int from = src[base + min(u.row, count - 1)], tensor = u.tensor & 1;       // (a valid row without a condition)
        const llla_strides &ss = tensor ? a.sv : a.sk;
        w[it] = *reinterpret_cast<const uint4 *>(static_cast<const int8_t *>(tensor ? a.V : a.K) + b * ss.batch + h * ss.head +
                                                 (int64_t)from * ss.seq + 16 * u.part);
        e0[it] = (tensor ? a.ve : a.ke)[exps + from / CACHE_BLOCK];
        const int n = mine ? exponent_needed<F>(w[it], e0[it]) : EXP_LEAST;
        need[0] = tensor ? need[0] : exponent_join(need[0], n);
        need[1] = tensor ? exponent_join(need[1], n) : need[1];
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        need[t] = wave_join(need[t]);
        if (tid % 64 == 0) needs[t][tid / 64] = need[t];
    }
    __syncthreads();
    int now[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) now[t] = exponent_join(exponent_join(needs[t][0], needs[t][1]), exponent_join(needs[t][2], needs[t][3]));
    if (tid < 2) (tid ? a.ved : a.ked)[(size_t)bh * cache_blocks(a.Ld_max) + blk] = (int8_t)(tid ? now[1] : now[0]);
#pragma unroll
    for (int it = 0; it < U::ITER; ++it) {
        const U u(it, tid);
        if ((U::PARTIAL && tid >= U::ALL) || u.row >= count) continue;
        const int e = u.tensor ? now[1] : now[0];
        const llla_strides &ds = u.tensor ? a.dv : a.dk;
        *reinterpret_cast<uint4 *>(static_cast<int8_t *>(u.tensor ? a.Vd : a.Kd) + b * ds.batch + h * ds.head + (int64_t)(base + u.row) * ds.seq + 16 * u.part) =
            e == EXP_NAN || e == e0[it] ? w[it] : shift16<F>(w[it], e0[it], e);
    }
}

// Rows of codes in place: one wave per block of destinations, most of which have few holes or none (256 heads x 64 rows into 4096 slots 10 us).  In these moments the block that holds slot
// `keep` may be getting another exponent; rows that come from it take the one that the plan saw.
template <int D, typename F>
__global__ __launch_bounds__(NT) void fill_holes_kernel(MoveArgs a)
{
    constexpr int PER_ROW = D / 16, AT_ONCE = 64 / (2 * PER_ROW);      // lanes of a row of one tensor; holes of a round
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int bh = blockIdx.y, b = bh / a.H, h = bh % a.H, blk = blockIdx.x * (NT / 64) + wave, base = blk * CACHE_BLOCK;
    if (blk >= a.plan.blocks) return;
    const int *hdr = a.ws + (size_t)bh * a.plan.words, *src = hdr + PLAN_HDR, *dst = src + a.plan.most, *hole_of = dst + a.plan.most;
    const int i0 = __builtin_amdgcn_readfirstlane(hole_of[blk]), count = __builtin_amdgcn_readfirstlane(hole_of[blk + 1]) - i0;
    if (count <= 0) return;
    const int mine = i0 + min(lane, count - 1), from = src[mine], to = dst[mine];         // of hole `lane`
    const size_t exps = (size_t)bh * cache_blocks(a.L_max);
    const int tensor = lane / (32), hole = lane % 32 / PER_ROW, part = lane % PER_ROW;
    const llla_strides &s = tensor ? a.sv : a.sk;
    int8_t *X = static_cast<int8_t *>(tensor ? a.Vd : a.Kd) + b * s.batch + h * s.head;
    const int8_t *exp = tensor ? a.ve : a.ke;
    const int was = exp[exps + blk];
    int need = EXP_LEAST;
    for (int i = 0; i < count; i += AT_ONCE) {
        const int f = __shfl(from, min(i + hole, count - 1)), fb = f / CACHE_BLOCK;
        const uint4 w = *reinterpret_cast<const uint4 *>(X + (int64_t)f * s.seq + 16 * part);
        const int e = fb == a.keep / CACHE_BLOCK ? hdr[1 + tensor] : (int)exp[exps + fb];
        need = exponent_join(need, exponent_needed<F>(w, e));
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) need = exponent_join(need, __shfl_xor(need, off));      // over the 32 lanes of a tensor
    const int now = exponent_join(was, need);
    if (now != was && now != EXP_NAN)                     // (rare) the rows that are there
        for (int r = hole; r < CACHE_BLOCK; r += AT_ONCE)
            if (base + r < a.keep) {
                uint4 *p = reinterpret_cast<uint4 *>(X + (int64_t)(base + r) * s.seq + 16 * part);
                *p = shift16<F>(*p, was, now);
            }
    for (int i = 0; i < count; i += AT_ONCE) {
        const int f = __shfl(from, min(i + hole, count - 1)), t = __shfl(to, min(i + hole, count - 1)), fb = f / CACHE_BLOCK;
        const uint4 w = *reinterpret_cast<const uint4 *>(X + (int64_t)f * s.seq + 16 * part);
        const int e = fb == a.keep / CACHE_BLOCK ? hdr[1 + tensor] : (int)exp[exps + fb];
        if (i + hole < count)
            *reinterpret_cast<uint4 *>(X + (int64_t)t * s.seq + 16 * part) = now == EXP_NAN || now == e ? w : shift16<F>(w, e, now);
    }
    if (lane % 32 == 0) (tensor ? a.ved : a.ked)[exps + blk] = (int8_t)now;
    if (lane < count) move_row_words(a, bh, from, to);
}

template <int D>
hipError_t launch_moves(const EvictProblem &p, MoveArgs a)
{
    const int bh = p.c.B * p.c.H, size = p.c.type == LLLA_F32 ? 4 : p.c.type == LLLA_BF16 ? 2 : 1;
    if (size == 1) {
        const int blocks = cache_blocks(p.keep);
        const dim3 grid(p.in_place ? (blocks + NT / 64 - 1) / (NT / 64) : blocks, bh);
        const bool i8 = p.c.type == LLLA_I8;
        if (p.in_place && i8) hipLaunchKernelGGL((fill_holes_kernel<D, Int8Code>), grid, dim3(NT), 0, p.stream, a);
        else if (p.in_place) hipLaunchKernelGGL((fill_holes_kernel<D, E4m3Code>), grid, dim3(NT), 0, p.stream, a);
        else if (i8) hipLaunchKernelGGL((move_codes_kernel<D, Int8Code>), grid, dim3(NT), 0, p.stream, a);
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
    else if (c.L_max <= 4096) hipLaunchKernelGGL((evict_plan_kernel<1024, 4>), grid, dim3(1024), 0, p.stream, a);
    else if (c.L_max <= 8192) hipLaunchKernelGGL((evict_plan_kernel<1024, 8>), grid, dim3(1024), 0, p.stream, a);
    else if (c.L_max <= ONE_LAUNCH) hipLaunchKernelGGL((evict_plan_kernel<1024, 16>), grid, dim3(1024), 0, p.stream, a);
    else
        for (int step = 0; step <= 5; ++step) hipLaunchKernelGGL(evict_long_kernel, dim3(plan.chunks, bh), dim3(NT), 0, p.stream, a, step);
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
