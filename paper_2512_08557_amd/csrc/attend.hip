// Attention of a call's new tokens over the token cache: how a call is cut up, and
// the entry points.  The kernels are in attend_kernel.h.
#include "attend_kernel.h"

#include <algorithm>
#include <cmath>
#include <limits>

namespace ssc {

namespace {

bool attend_cut(const sscater_attend_spec* s, const sscater_token_cache* c, const sscater_token_rows* r, AttendCut* cut) {
    if (!s || !token_cache_ok(c) || !token_rows_ok(c, r)) return false;
    if (s->q_heads < 1 || s->q_heads > (1 << 16) || s->q_heads % c->kv_heads || s->window < 1 || s->causal < 0 ||
        s->causal > 1 || !(s->scale == s->scale))
        return false;
    const int64_t reach = std::min((int64_t)s->window + r->max_new - 1, r->max_past + r->max_new);
    if (r->tokens > 0 && c->capacity - c->sinks < reach) return false;
    const int64_t rows = (int64_t)r->max_new * (s->q_heads / c->kv_heads);
    if (rows > (1 << 30) || (int64_t)r->tokens * s->q_heads > (int64_t(1) << 40)) return false;
    cut_keys(cut, c->dtype == SSCATER_F32, c->head_dim, rows, (int64_t)c->kv_heads * c->batch, reach + c->sinks, false);
    return cut->grid <= 0x7FFFFFFF;
}

size_t attend_bytes(const AttendCut& cut, const sscater_attend_spec* s, const sscater_token_cache* c,
                    const sscater_token_rows* r) {
    return cut.splits > 1 ? (size_t)cut.splits * r->tokens * s->q_heads * (c->head_dim + 2) * 4 : 0;
}

template <bool F32, int D>
void launch_attend(AttendArgs a, const AttendCut& cut, hipStream_t s) {
    const dim3 block(256);
    for (int64_t at = 0; at < cut.grid; at += LAUNCH_GROUPS) {
        a.id0 = (int)at;
        const dim3 grid((unsigned)std::min(LAUNCH_GROUPS, cut.grid - at));
        if constexpr (!(F32 && D == 128)) {
            if (cut.wm == 1) attend_kernel<F32, D, 1, Keys::CACHE, false><<<grid, block, 0, s>>>(a);
        }
        if (cut.wm == 2) attend_kernel<F32, D, 2, Keys::CACHE, !F32><<<grid, block, 0, s>>>(a);
        if (cut.wm == 4) attend_kernel<F32, D, 4, Keys::CACHE, !F32><<<grid, block, 0, s>>>(a);
    }
    if (cut.splits > 1) {                              // at most some hundred thousand rows: see cut_keys
        const int64_t rows = (int64_t)a.rows.tokens * a.q_heads;
        join_kernel<F32, D, true><<<dim3((unsigned)((rows + 3) / 4)), block, 0, s>>>(a.part, a.out, rows, cut.splits,
                                                                                     a.q_heads, rows_end(a.rows));
    }
}

template <bool F32>
void launch_attend(const AttendArgs& a, const AttendCut& cut, int dim, hipStream_t s) {
    if (dim == 32) launch_attend<F32, 32>(a, cut, s);
    else if (dim == 64) launch_attend<F32, 64>(a, cut, s);
    else launch_attend<F32, 128>(a, cut, s);
}

}  // namespace

}  // namespace ssc

using namespace ssc;

extern "C" {

int sscater_tokens_workspace(const sscater_attend_spec* spec, const sscater_token_cache* cache,
                             const sscater_token_rows* rows, size_t* bytes) {
    AttendCut cut;
    if (!bytes || !attend_cut(spec, cache, rows, &cut)) return SSCATER_E_INVALID_ARG;
    *bytes = attend_bytes(cut, spec, cache, rows);
    return SSCATER_OK;
}

int sscater_tokens_attend(const sscater_attend_spec* spec, const sscater_token_cache* cache,
                          const sscater_token_rows* rows, const void* q, void* out, void* workspace,
                          size_t workspace_bytes, void* stream) {
    AttendCut cut;
    if (!attend_cut(spec, cache, rows, &cut)) return SSCATER_E_INVALID_ARG;
    if (rows->tokens == 0) return SSCATER_OK;
    const size_t need = attend_bytes(cut, spec, cache, rows);
    if (!q || !out || (uintptr_t)q % 16 || (uintptr_t)out % 16) return SSCATER_E_INVALID_ARG;
    if (need > 0 && (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < need)) return SSCATER_E_INVALID_ARG;
    AttendArgs a;
    a.rows = token_rows(cache, rows);
    a.q = q; a.k = cache->k; a.v = cache->v; a.out = out; a.part = (float*)workspace;
    a.q_heads = spec->q_heads; a.kv_heads = cache->kv_heads; a.group = spec->q_heads / cache->kv_heads;
    a.sinks = cache->sinks; a.capacity = cache->capacity; a.window = spec->window; a.causal = spec->causal;
    a.qtiles = cut.qtiles; a.splits = cut.splits;
    // not zero, so that a masked score times it stays -inf; the least number of all, times a finite score, is zero beside 1
    a.scale = std::max(std::fabs(spec->scale) * 1.4426950408889634f, std::numeric_limits<float>::denorm_min());
    a.flip = spec->scale < 0.f ? cache->dtype == SSCATER_F32 ? 0x80000000u : 0x80008000u : 0u;
    if (cache->dtype == SSCATER_F32) launch_attend<true>(a, cut, cache->head_dim, (hipStream_t)stream);
    else launch_attend<false>(a, cut, cache->head_dim, (hipStream_t)stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSCATER_OK : report_hip_error(e);
}

}  // extern "C"
