// C ABI of the cache calls: host-side validation.  Every check runs before anything is enqueued.
#include <cmath>

#include "llla_cache.hpp"

namespace {

bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
int size_of(llla_dtype t) { return t == LLLA_F32 ? 4 : t == LLLA_BF16 ? 2 : 1; }
bool codes(llla_dtype t) { return t == LLLA_I8 || t == LLLA_E4M3; }
bool number_type(llla_dtype t) { return t == LLLA_F32 || t == LLLA_BF16; }
bool dim_ok(int d) { return d == 16 || d == 32 || d == 64 || d == 128; }

bool strides_cover(const llla_strides &s, int B, int H, int64_t n, int d)
{
    if (s.head < 0 || s.batch < 0 || s.seq < 0) return false;
    return !((s.seq < d && n > 1) || (H > 1 && s.head == 0) || (B > 1 && s.batch == 0));
}
bool strides_aligned(const llla_strides &s, llla_dtype t)
{
    const int64_t q = 16 / size_of(t);
    return s.batch % q == 0 && s.head % q == 0 && s.seq % q == 0;
}

constexpr int64_t MAX_ROW_STRIDE = (int64_t)1 << 25;      // elements: offsets of 64 rows are kept in 32 bits

// values: whether V is used
llla_status check_cache(const llla_cache *c, bool values)
{
    if (!c || !c->K || (values && !c->V)) return LLLA_ERR_NULL;
    if (c->B <= 0 || c->H <= 0 || c->L_max <= 0 || c->d <= 0) return LLLA_ERR_SHAPE;
    if (!number_type(c->type) && !codes(c->type)) return LLLA_ERR_DTYPE;
    if (!dim_ok(c->d)) return LLLA_ERR_UNSUPPORTED;
    if (codes(c->type) && (!c->k_exp || (values && !c->v_exp))) return LLLA_ERR_NULL;
    if ((int64_t)c->B * c->H > 65535 || c->L_max > (1 << 30)) return LLLA_ERR_SHAPE;
    if (!strides_cover(c->sk, c->B, c->H, c->L_max, c->d) || (values && !strides_cover(c->sv, c->B, c->H, c->L_max, c->d))) return LLLA_ERR_SHAPE;
    if (c->sk.seq >= MAX_ROW_STRIDE || (values && c->sv.seq >= MAX_ROW_STRIDE)) return LLLA_ERR_SHAPE;
    if (!aligned(c->K, 16) || !strides_aligned(c->sk, c->type) || (values && (!aligned(c->V, 16) || !strides_aligned(c->sv, c->type))) ||
        !aligned(c->scores, 4) || !aligned(c->pos, 4))
        return LLLA_ERR_ALIGN;
    return LLLA_OK;
}

// keys and values of a cache that is written must be two arrays
bool twice(const llla_cache &c) { return c.K == c.V || (codes(c.type) && c.k_exp == c.v_exp); }

llla_status check_workspace(size_t need, const void *ws, size_t bytes)
{
    if (need == 0) return LLLA_OK;
    return ws == nullptr || bytes < need || !aligned(ws, 256) ? LLLA_ERR_WORKSPACE : LLLA_OK;
}

}  // namespace

extern "C" {

llla_status llla_cache_append(const llla_cache *cache, const void *k, const void *v, llla_strides sk, llla_strides sv, int n,
                              llla_dtype in, const int32_t *seqlens, const int32_t *new_lens, const int32_t *first_pos,
                              void *stream)
{
    if (!k || !v) return LLLA_ERR_NULL;
    llla_status st = check_cache(cache, true);
    if (st != LLLA_OK) return st;
    if (n <= 0) return LLLA_ERR_SHAPE;
    if (!number_type(in)) return LLLA_ERR_DTYPE;
    if (twice(*cache)) return LLLA_ERR_PARAM;
    if (!strides_cover(sk, cache->B, cache->H, n, cache->d) || !strides_cover(sv, cache->B, cache->H, n, cache->d)) return LLLA_ERR_SHAPE;
    if (!aligned(k, 16) || !aligned(v, 16) || !strides_aligned(sk, in) || !strides_aligned(sv, in) || !aligned(seqlens, 4) ||
        !aligned(new_lens, 4) || !aligned(first_pos, 4))
        return LLLA_ERR_ALIGN;
    llla::AppendProblem p{*cache, k, v, sk, sv, n, in, seqlens, new_lens, first_pos, static_cast<hipStream_t>(stream)};
    return llla::cache_append(p) == hipSuccess ? LLLA_OK : LLLA_ERR_LAUNCH;
}

size_t llla_decode_q8_workspace_bytes(const llla_cache *c, int H)
{
    if (!c || c->B <= 0 || c->H <= 0 || H <= 0 || H % c->H != 0 || (int64_t)c->B * H > 65535 || c->L_max <= 0 || !dim_ok(c->d) || !codes(c->type)) return 0;
    return llla::decode_q8_workspace_bytes(c->B, H, c->L_max, c->d);
}

llla_status llla_decode_q8(const void *q, const llla_cache *cache, void *o, const int32_t *seqlens, int H,
                           llla_dtype in, llla_dtype out, float lambda, float scale,
                           void *workspace, size_t workspace_bytes, void *stream)
{
    if (!q || !o) return LLLA_ERR_NULL;
    llla_status st = check_cache(cache, true);
    if (st != LLLA_OK) return st;
    if (!codes(cache->type) || !number_type(in) || !number_type(out)) return LLLA_ERR_DTYPE;
    if (H <= 0 || H % cache->H != 0 || (int64_t)cache->B * H > 65535) return LLLA_ERR_SHAPE;
    if (!(lambda > 0.f) || !std::isfinite(lambda) || !std::isfinite(scale)) return LLLA_ERR_PARAM;
    if (!aligned(q, 16) || !aligned(o, 16) || !aligned(seqlens, 4)) return LLLA_ERR_ALIGN;
    llla::DecodeQ8Problem p{*cache, q, o, seqlens, H, in, out, lambda, scale, workspace, workspace_bytes, static_cast<hipStream_t>(stream)};
    llla::stage_begin(p.stream);
    const hipError_t e = llla::decode_q8(p);
    llla::stage_end(p.stream);
    return e == hipSuccess ? LLLA_OK : LLLA_ERR_LAUNCH;
}

size_t llla_cache_scores_workspace_bytes(const llla_cache *c, int H, int nq, llla_dtype in)
{
    if (!c || c->B <= 0 || c->H <= 0 || H <= 0 || H % c->H != 0 || nq <= 0 || c->L_max <= 0 || !dim_ok(c->d) || !number_type(in)) return 0;
    return llla::cache_scores_workspace_bytes(*c, H, nq, in);
}

llla_status llla_cache_scores(const void *Q, const llla_cache *cache, llla_strides sq, const int32_t *seqlens, int H, int nq,
                              llla_dtype in, float scale, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!Q) return LLLA_ERR_NULL;
    llla_status st = check_cache(cache, false);
    if (st != LLLA_OK) return st;
    if (!cache->scores) return LLLA_ERR_NULL;
    if (!number_type(in) || (!codes(cache->type) && cache->type != in)) return LLLA_ERR_DTYPE;
    if (H <= 0 || nq <= 0 || H % cache->H != 0 || (int64_t)cache->B * H > 65535) return LLLA_ERR_SHAPE;
    if ((int64_t)H / cache->H * nq > 2147483647LL - 1024 || !strides_cover(sq, cache->B, H, nq, cache->d)) return LLLA_ERR_SHAPE;
    if (!std::isfinite(scale)) return LLLA_ERR_PARAM;
    if (!aligned(Q, 16) || !strides_aligned(sq, in) || !aligned(seqlens, 4)) return LLLA_ERR_ALIGN;
    st = check_workspace(llla::cache_scores_workspace_bytes(*cache, H, nq, in), workspace, workspace_bytes);
    if (st != LLLA_OK) return st;
    llla::ScoresProblem p{*cache, Q, sq, seqlens, H, nq, in, scale, workspace, static_cast<hipStream_t>(stream)};
    return llla::cache_scores(p) == hipSuccess ? LLLA_OK : LLLA_ERR_LAUNCH;
}

size_t llla_cache_evict_workspace_bytes(const llla_cache *c, int keep)
{
    if (!c || c->B <= 0 || c->H <= 0 || c->L_max <= 0 || keep <= 0 || keep > c->L_max) return 0;
    return llla::cache_evict_workspace_bytes(*c, keep);
}

llla_status llla_cache_evict(const llla_cache *cache, const llla_cache *into, const int32_t *seqlens, int keep, int sinks,
                             int recent, int32_t *lens, int32_t *index, void *workspace, size_t workspace_bytes, void *stream)
{
    llla_status st = check_cache(cache, true);
    if (st != LLLA_OK) return st;
    if (!cache->scores || !lens) return LLLA_ERR_NULL;
    if (keep <= 0 || keep > cache->L_max) return LLLA_ERR_SHAPE;
    if (sinks < 0 || recent < 0 || (int64_t)sinks + recent > keep || lens == seqlens || (!into && twice(*cache))) return LLLA_ERR_PARAM;
    if (into) {
        st = check_cache(into, true);
        if (st != LLLA_OK) return st;
        if (into->B != cache->B || into->H != cache->H || into->d != cache->d || into->L_max < keep) return LLLA_ERR_SHAPE;
        if (into->type != cache->type) return LLLA_ERR_DTYPE;
        if (into->K == cache->K || into->V == cache->V || into->K == cache->V || into->V == cache->K || twice(*into) || (into->scores && into->scores == cache->scores) ||
            (into->pos && into->pos == cache->pos) || (codes(cache->type) && (into->k_exp == cache->k_exp || into->v_exp == cache->v_exp)))
            return LLLA_ERR_PARAM;
    }
    if (!aligned(seqlens, 4) || !aligned(lens, 4) || !aligned(index, 4)) return LLLA_ERR_ALIGN;
    st = check_workspace(llla::cache_evict_workspace_bytes(*cache, keep), workspace, workspace_bytes);
    if (st != LLLA_OK) return st;
    llla::EvictProblem p{*cache, into ? *into : *cache, into == nullptr, seqlens, keep, sinks, recent, lens, index, workspace,
                         static_cast<hipStream_t>(stream)};
    return llla::cache_evict(p) == hipSuccess ? LLLA_OK : LLLA_ERR_LAUNCH;
}

}  // extern "C"
