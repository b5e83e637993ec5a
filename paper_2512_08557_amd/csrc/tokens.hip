// Heads of the new tokens into queries and the token cache, and the streams'
// lengths.
//
// One pass over the projected rows: a workgroup takes TT tokens, forms the
// cosines and sines of their angles once for all heads in LDS, and then goes
// through the tokens' heads, a head by G lanes with two 16-byte pieces each
// (the same places of both halves of the head), whose sum of squares is
// reduced between those lanes.  Every value is read and written once: 60055 fp32
// tokens of 8 query and 4 key heads of 64 values 95 us, 5.2 TB/s, the rate of a
// copy; one token 3.6 us, a launch, the positions' and the row's round trips.
//
// The angle in turns is position * inv_freq / (2 pi) in 64 bits less its whole
// part: a stream's stride number passes 10^6 within hours, where 32 bits would
// be off by 0.06 radians.
#include "tokens.h"

#include <algorithm>

namespace ssc {

struct AppendArgs {
    TokenRows rows;
    const void* qkv;
    const void* qw;
    const void* kw;
    const float* inv_freq;
    const int32_t* pos;
    void* q;
    void* k;
    void* v;
    int64_t ld;
    int q_heads, kv_heads, axes, sinks, capacity, even;
    int end0, end1;        // pairs of the first axis, and of the first two
    int tt;                // tokens of a workgroup
    int token0;            // first token of the launch
    float eps;
};

constexpr int APPEND_TOKENS = 4;      // at most per workgroup

// Sixteen bytes of values as fp32, and back.
template <bool F32>
struct Piece {
    static constexpr int E = F32 ? 4 : 8;
    float v[E];
    __device__ __forceinline__ void unpack(const uint4 u) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (F32) v[i] = __uint_as_float(w[i]);
            else {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        }
    }
    __device__ __forceinline__ uint4 pack() const {
        if constexpr (F32)
            return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        else
            return make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
    }
};

// 16 bytes from an address that may be aligned to its elements only
template <bool VEC>
__device__ __forceinline__ uint4 load16(const char* p) {
    if constexpr (VEC) return *(const uint4*)p;
    uint4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

template <bool F32, int D, bool VEC>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
    constexpr int S = F32 ? 4 : 2, E = 16 / S;
    constexpr int G = D / (2 * E);                   // lanes of a head
    __shared__ float2 turn[APPEND_TOKENS][D / 2];
    __shared__ int64_t slot[APPEND_TOKENS];           // cache row of the token's first head, or -1
    const int t0 = a.token0 + (int)blockIdx.x * a.tt;
    const int nt = min(a.tt, a.rows.tokens - t0);
    for (int i = threadIdx.x; i < nt * (D / 2); i += 256) {
        const int t = i / (D / 2), p = i % (D / 2);
        const int axis = p < a.end0 ? 0 : p < a.end1 ? 1 : 2;
        const double turns = (double)a.pos[(int64_t)(t0 + t) * a.axes + axis] * a.inv_freq[p] * 0.15915494309189535;
        const float f = (float)(turns - rint(turns));
        float sn, cs;
        sincospif(2.f * f, &sn, &cs);
        turn[t][p] = make_float2(cs, sn);
    }
    if ((int)threadIdx.x < nt) {
        const int row = t0 + threadIdx.x;
        // the sequence: the last whose first row is not after this one
        int b;
        if (a.rows.start) {
            int lo = 0, hi = a.rows.batch - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (a.rows.start[mid] <= row) lo = mid; else hi = mid - 1;
            }
            b = lo;
        } else {
            b = row / a.rows.max_new;
        }
        int first, n;
        rows_of(a.rows, b, first, n);
        int64_t at = -1;
        if (row >= first && row - first < n) {
            const int ring = a.capacity - a.sinks;
            const int64_t past = past_of(a.rows, b), j = past + (row - first);
            if (j < a.sinks) at = j;
            else if (j >= past + n - ring) at = a.sinks + (j - a.sinks) % ring;
            if (at >= 0) at += (int64_t)b * a.kv_heads * a.capacity;
        }
        slot[threadIdx.x] = at;
    }
    __syncthreads();
    const int heads = a.q_heads + 2 * a.kv_heads;
    const int sub = threadIdx.x % G;
    const int items = nt * heads;
    // every lane goes round as often as the first, for the reductions
    for (int it0 = 0; it0 < items; it0 += 256 / G) {
        const int it = it0 + (int)threadIdx.x / G;
        const bool live = it < items;
        const int t = live ? it / heads : 0, hd = live ? it % heads : 0;
        const char* src = (const char*)a.qkv + ((int64_t)(t0 + t) * a.ld + (int64_t)hd * D) * S;
        uint4 lo = load16<VEC>(src + sub * 16), hi = load16<VEC>(src + D / 2 * S + sub * 16);
        const bool key = hd >= a.q_heads, value = hd >= a.q_heads + a.kv_heads;
        Piece<F32> x, y;
        x.unpack(lo);
        y.unpack(hi);
        const void* weight = key ? a.kw : a.qw;
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) ss = fmaf(x.v[e], x.v[e], fmaf(y.v[e], y.v[e], ss));
#pragma unroll
        for (int o = 1; o < G; o <<= 1) ss += __shfl_xor(ss, o);
        if (!value) {
            if (weight) {
                const float r = 1.f / sqrtf(ss * (1.f / D) + a.eps);
                Piece<F32> wx, wy;
                wx.unpack(load16<false>((const char*)weight + sub * 16));
                wy.unpack(load16<false>((const char*)weight + D / 2 * S + sub * 16));
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    x.v[e] = x.v[e] * r * wx.v[e];
                    y.v[e] = y.v[e] * r * wy.v[e];
                }
            }
            if (a.even) {
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const float2 c = turn[t][sub * (E / 2) + e / 2], d = turn[t][D / 4 + sub * (E / 2) + e / 2];
                    const float x0 = x.v[e], y0 = y.v[e];
                    x.v[e] = x0 * c.x - x.v[e + 1] * c.y;
                    x.v[e + 1] = x0 * c.y + x.v[e + 1] * c.x;
                    y.v[e] = y0 * d.x - y.v[e + 1] * d.y;
                    y.v[e + 1] = y0 * d.y + y.v[e + 1] * d.x;
                }
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float2 c = turn[t][sub * E + e];
                    const float x0 = x.v[e];
                    x.v[e] = x0 * c.x - y.v[e] * c.y;
                    y.v[e] = x0 * c.y + y.v[e] * c.x;
                }
            }
            lo = x.pack();
            hi = y.pack();
        }
        if (!live) continue;
        char* dst;
        if (!key) {
            dst = (char*)a.q + ((int64_t)(t0 + t) * a.q_heads + hd) * (D * S);
        } else {
            if (slot[t] < 0) continue;
            const int h = hd - a.q_heads - (value ? a.kv_heads : 0);
            dst = (char*)(value ? a.v : a.k) + (slot[t] + (int64_t)h * a.capacity) * (D * S);
        }
        *(uint4*)(dst + sub * 16) = lo;
        *(uint4*)(dst + D / 2 * S + sub * 16) = hi;
    }
}

__global__ __launch_bounds__(256) void advance_kernel(TokenRows rows, int64_t* past) {
    const int b = blockIdx.x * 256 + threadIdx.x;
    if (b >= rows.batch) return;
    int first, n;
    rows_of(rows, b, first, n);
    past[b] = past_of(rows, b) + n;
}

bool token_cache_ok(const sscater_token_cache* c) {
    if (!c || (c->dtype != SSCATER_F32 && c->dtype != SSCATER_BF16)) return false;
    if (c->batch < 1 || c->batch > (1 << 24) || c->kv_heads < 1 || c->kv_heads > (1 << 16)) return false;
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return false;
    if (c->sinks < 0 || c->capacity <= c->sinks || c->capacity > (1 << 30)) return false;
    for (const void* p : {c->k, c->v})
        if (!p || (uintptr_t)p % 16) return false;
    return c->past && (uintptr_t)c->past % 8 == 0;
}

bool token_rows_ok(const sscater_token_cache* c, const sscater_token_rows* r) {
    if (!r || r->tokens < 0 || r->tokens > (1 << 30) || r->max_new < 0 || r->max_new > r->tokens) return false;
    if (r->max_past < 0 || r->max_past > (int64_t(1) << 62)) return false;
    if (r->tokens > 0 && r->max_new < 1) return false;
    if (!r->start && (int64_t)r->max_new * c->batch != r->tokens) return false;
    return (int64_t)r->max_new * c->batch >= r->tokens && (uintptr_t)r->start % 4 == 0;
}

TokenRows token_rows(const sscater_token_cache* c, const sscater_token_rows* r) {
    TokenRows t;
    t.tokens = r->tokens;
    t.max_new = r->max_new;
    t.batch = c->batch;
    t.start = r->start;
    t.past = c->past;
    return t;
}

namespace {

template <bool F32, int D>
void launch_append(AppendArgs a, bool vec, hipStream_t s) {
    for (int64_t t = 0; t < a.rows.tokens; t += LAUNCH_GROUPS * a.tt) {
        a.token0 = (int)t;
        const dim3 grid((unsigned)std::min(LAUNCH_GROUPS, (a.rows.tokens - t + a.tt - 1) / a.tt)), block(256);
        if (vec) append_kernel<F32, D, true><<<grid, block, 0, s>>>(a);
        else append_kernel<F32, D, false><<<grid, block, 0, s>>>(a);
    }
}

template <bool F32>
void launch_append(const AppendArgs& a, int dim, bool vec, hipStream_t s) {
    if (dim == 32) launch_append<F32, 32>(a, vec, s);
    else if (dim == 64) launch_append<F32, 64>(a, vec, s);
    else launch_append<F32, 128>(a, vec, s);
}

}  // namespace

}  // namespace ssc

using namespace ssc;

extern "C" {

int sscater_tokens_append(const sscater_head_spec* spec, const sscater_token_cache* cache,
                          const sscater_token_rows* rows, const void* qkv, const void* q_weight, const void* k_weight,
                          const float* inv_freq, const int32_t* pos, void* q, void* stream) {
    if (!spec || !token_cache_ok(cache) || !token_rows_ok(cache, rows)) return SSCATER_E_INVALID_ARG;
    const int D = cache->head_dim, size = cache->dtype == SSCATER_F32 ? 4 : 2;
    if (spec->q_heads < 1 || spec->q_heads > (1 << 16) || spec->axes < 1 || spec->axes > 3 || spec->interleaved < 0 ||
        spec->interleaved > 1 || !(spec->eps >= 0.f))
        return SSCATER_E_INVALID_ARG;
    int pairs = 0;
    for (int i = 0; i < spec->axes; ++i) {
        if (spec->section[i] < 0 || spec->section[i] > D / 2) return SSCATER_E_INVALID_ARG;
        pairs += spec->section[i];
    }
    if (pairs != D / 2) return SSCATER_E_INVALID_ARG;
    const int64_t width = ((int64_t)spec->q_heads + 2 * (int64_t)cache->kv_heads) * D;
    if (spec->qkv_stride < width || width > (1 << 30)) return SSCATER_E_INVALID_ARG;
    if ((q_weight == nullptr) != (k_weight == nullptr)) return SSCATER_E_INVALID_ARG;
    if (rows->tokens == 0) return SSCATER_OK;
    for (const void* p : {qkv, (const void*)inv_freq, (const void*)pos, (const void*)q})
        if (!p) return SSCATER_E_INVALID_ARG;
    if ((uintptr_t)qkv % size || (uintptr_t)q_weight % size || (uintptr_t)k_weight % size ||
        (uintptr_t)inv_freq % 4 || (uintptr_t)pos % 4 || (uintptr_t)q % 16)
        return SSCATER_E_INVALID_ARG;
    AppendArgs a;
    a.rows = token_rows(cache, rows);
    a.qkv = qkv; a.qw = q_weight; a.kw = k_weight; a.inv_freq = inv_freq; a.pos = pos;
    a.q = q; a.k = cache->k; a.v = cache->v;
    a.ld = spec->qkv_stride;
    a.q_heads = spec->q_heads; a.kv_heads = cache->kv_heads; a.axes = spec->axes;
    a.sinks = cache->sinks; a.capacity = cache->capacity; a.even = spec->interleaved;
    a.end0 = spec->section[0];
    a.end1 = spec->axes > 1 ? spec->section[0] + spec->section[1] : D / 2;
    a.eps = spec->eps;
    // tokens of a workgroup: enough workgroups for the card, then longer ones (8 query and 4 key heads of 64 values, one,
    // two, four and eight tokens: 100000 bf16 tokens 204 us, 119, 80, 80; 100000 in fp32 209, 142, 146, 153; 13000 in fp32
    // 23.5, 19.6, 17.9, 18.7)
    a.tt = std::min(APPEND_TOKENS, std::max(1, rows->tokens / 1024));
    const bool vec = (uintptr_t)qkv % 16 == 0 && a.ld * size % 16 == 0;
    if (size == 4) launch_append<true>(a, D, vec, (hipStream_t)stream);
    else launch_append<false>(a, D, vec, (hipStream_t)stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSCATER_OK : report_hip_error(e);
}

int sscater_tokens_advance(const sscater_token_cache* cache, const sscater_token_rows* rows, void* stream) {
    if (!token_cache_ok(cache) || !token_rows_ok(cache, rows)) return SSCATER_E_INVALID_ARG;
    if (rows->tokens == 0) return SSCATER_OK;
    advance_kernel<<<dim3((cache->batch + 255) / 256), dim3(256), 0, (hipStream_t)stream>>>(token_rows(cache, rows),
                                                                                            cache->past);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSCATER_OK : report_hip_error(e);
}

}  // extern "C"
