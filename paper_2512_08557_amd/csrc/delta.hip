// The gated delta rule: a memory of fixed size for every stream and head, a matrix
// S [key_dim][value_dim] in fp32 that is read and corrected by every token:
//
//   u = beta (v - alpha S^T k),  S = alpha S + k u^T,  o = scale S^T q
//
// Tokens one by one: a wavefront owns 32 columns of a head's state in its registers
// (columns do not depend on one another).  Lane 8 c + r holds the r-th eighth of the
// rows of columns 4 c .. 4 c + 3, so a product with the state is key_dim / 2
// multiplications a lane and a sum between eight neighbouring lanes, and q and k come
// as one run of values for each lane.
#include "tokens.h"

#include <algorithm>

namespace ssc {

struct DeltaArgs {
    TokenRows rows;
    const float* from;     // the states before
    float* state;
    const void* q;
    const void* k;
    const void* v;
    const void* a;
    const void* b;
    const float* rate;
    const float* bias;
    void* out;
    int64_t ldq, ldk, ldv, lda, ldb;
    int64_t item0;         // first wavefront of the launch
    int heads, group;      // value heads, and those that share a query and key head
    int unit;
    float eps, scale;
};

template <bool F32>
__device__ __forceinline__ float value_at(const void* p, int64_t i) {
    if constexpr (F32) return ((const float*)p)[i];
    return __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16);
}

// N neighbouring values, aligned to themselves only.
template <bool F32, int N>
__device__ __forceinline__ void values_at(const void* p, int64_t i, float (&v)[N]) {
    if constexpr (F32) {
        __builtin_memcpy(v, (const float*)p + i, 4 * N);
    } else {
        uint32_t u[N / 2];
        __builtin_memcpy(u, (const uint16_t*)p + i, 2 * N);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = __uint_as_float(e & 1 ? u[e / 2] & 0xFFFF0000u : u[e / 2] << 16);
    }
}

// The sum over eight neighbouring lanes, the same bits in all of them.
__device__ __forceinline__ float sum8(float v) {
    auto add = [&](auto ctrl) __attribute__((always_inline)) {
        constexpr int C = decltype(ctrl)::value;
        v += __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), C, 0xF, 0xF, true));
    };
    add(std::integral_constant<int, 0xB1>{});          // the neighbour
    add(std::integral_constant<int, 0x4E>{});          // the other pair of four
    add(std::integral_constant<int, 0x141>{});         // the other four of eight, back to front
    return v;
}

// log(alpha) and beta of a token.  Below -1000 alpha is zero by far.
__device__ __forceinline__ float log_alpha(float a, float rate, float bias, bool raw) {
    if (raw) {
        const float x = a + bias;
        a = -rate * (x > 20.f ? x : log1pf(expf(x)));
    }
    return a < -1000.f ? -1000.f : a;
}
__device__ __forceinline__ float beta_of(float b, bool raw) { return raw ? 1.f / (1.f + expf(-b)) : b; }

template <bool F32, int DK, int DV>
__global__ __launch_bounds__(256) void delta_token_kernel(DeltaArgs a) {
    constexpr int R = DK / 8, NB = DV / 32;
    const int lane = threadIdx.x & 63;
    const int64_t item = a.item0 + (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t which = item / NB;
    if (which >= (int64_t)a.rows.batch * a.heads) return;
    const int b = (int)(which / a.heads), h = (int)(which % a.heads), hk = h / a.group;
    int first, n;
    rows_of(a.rows, b, first, n);
    if (n == 0 && a.from == a.state) return;
    const int r0 = (lane & 7) * R, c0 = (int)(item % NB) * 32 + (lane >> 3) * 4;
    const int64_t at = (which * DK + r0) * DV + c0;
    f4v s[R];
#pragma unroll
    for (int i = 0; i < R; ++i) s[i] = *(const f4v*)(a.from + at + i * DV);
    const bool raw = a.rate != nullptr;
    const float rate = raw ? a.rate[h] : 0.f, bias = raw ? a.bias[h] : 0.f;
    struct Token {
        float q[R], k[R], v[4], a, b;
    };
    auto fetch = [&](int64_t t) __attribute__((always_inline)) {
        Token x;
        values_at<F32>(a.q, t * a.ldq + hk * DK + r0, x.q);
        values_at<F32>(a.k, t * a.ldk + hk * DK + r0, x.k);
        values_at<F32>(a.v, t * a.ldv + h * DV + c0, x.v);
        x.a = value_at<F32>(a.a, t * a.lda + h);
        x.b = value_at<F32>(a.b, t * a.ldb + h);
        return x;
    };
    Token next;
    if (n > 0) next = fetch(first);
    for (int i = 0; i < n; ++i) {
        const int64_t t = first + i;
        Token x = next;
        if (i + 1 < n) next = fetch(t + 1);
        float fq = a.scale, fk = 1.f;
        if (a.unit) {
            float qq = 0.f, kk = 0.f;
#pragma unroll
            for (int j = 0; j < R; ++j) {
                qq = fmaf(x.q[j], x.q[j], qq);
                kk = fmaf(x.k[j], x.k[j], kk);
            }
            fq *= 1.f / sqrtf(sum8(qq) + a.eps);
            fk = 1.f / sqrtf(sum8(kk) + a.eps);
        }
        const float alpha = expf(log_alpha(x.a, rate, bias, raw)), beta = beta_of(x.b, raw);
        f4v p = {0.f, 0.f, 0.f, 0.f}, o = {0.f, 0.f, 0.f, 0.f}, u;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            x.k[j] *= fk;
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = fmaf(s[j][e], x.k[j], p[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = beta * (x.v[e] - alpha * sum8(p[e]));
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[j][e] = fmaf(x.k[j], u[e], alpha * s[j][e]);
                o[e] = fmaf(s[j][e], x.q[j], o[e]);
            }
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = sum8(o[e]) * fq;
        if ((lane & 7) == 0) {
            const int64_t to = (t * a.heads + h) * DV + c0;
            if constexpr (F32) *(f4v*)((float*)a.out + to) = o;
            else *(uint2*)((uint16_t*)a.out + to) = make_uint2(bf16_pair(o[0], o[1]), bf16_pair(o[2], o[3]));
        }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) *(f4v*)(a.state + at + i * DV) = s[i];
}

namespace {

template <bool F32, int DK, int DV>
void launch_tokens(DeltaArgs a, hipStream_t s) {
    const int64_t groups = ((int64_t)a.rows.batch * a.heads * (DV / 32) + 3) / 4;
    for (int64_t g = 0; g < groups; g += LAUNCH_GROUPS) {
        a.item0 = g * 4;
        delta_token_kernel<F32, DK, DV><<<dim3((unsigned)std::min(LAUNCH_GROUPS, groups - g)), dim3(256), 0, s>>>(a);
    }
}

template <bool F32, int DK>
void launch_delta(const DeltaArgs& a, int dv, hipStream_t s) {
    if (dv == 32) launch_tokens<F32, DK, 32>(a, s);
    else if (dv == 64) launch_tokens<F32, DK, 64>(a, s);
    else launch_tokens<F32, DK, 128>(a, s);
}

template <bool F32>
void launch_delta(const DeltaArgs& a, int dk, int dv, hipStream_t s) {
    if (dk == 32) launch_delta<F32, 32>(a, dv, s);
    else if (dk == 64) launch_delta<F32, 64>(a, dv, s);
    else launch_delta<F32, 128>(a, dv, s);
}

bool head_size(int d) { return d == 32 || d == 64 || d == 128; }

bool delta_ok(const sscater_delta_spec* s, const sscater_delta_memory* m, const sscater_token_rows* r) {
    if (!s || !m || !r || (m->dtype != SSCATER_F32 && m->dtype != SSCATER_BF16)) return false;
    if (m->batch < 1 || m->batch > (1 << 24) || m->heads < 1 || m->heads > (1 << 16) || m->qk_heads < 1 ||
        m->heads % m->qk_heads || !head_size(m->key_dim) || !head_size(m->value_dim) || !m->state ||
        (uintptr_t)m->state % 16)
        return false;
    if (r->tokens < 0 || r->tokens > (1 << 30) || r->max_new < 0 || r->max_new > r->tokens ||
        (r->tokens > 0 && r->max_new < 1) || (!r->start && (int64_t)r->max_new * m->batch != r->tokens) ||
        (uintptr_t)r->start % 4)
        return false;
    const int64_t qk = (int64_t)m->qk_heads * m->key_dim, v = (int64_t)m->heads * m->value_dim;
    return s->unit >= 0 && s->unit <= 1 && s->eps >= 0.f && s->scale == s->scale && s->q_stride >= qk &&
           s->k_stride >= qk && s->v_stride >= v && s->a_stride >= m->heads && s->b_stride >= m->heads;
}

}  // namespace

}  // namespace ssc

using namespace ssc;

extern "C" {

int sscater_delta_workspace(const sscater_delta_spec* spec, const sscater_delta_memory* memory,
                            const sscater_token_rows* rows, size_t* bytes) {
    if (!bytes || !delta_ok(spec, memory, rows)) return SSCATER_E_INVALID_ARG;
    *bytes = 0;
    return SSCATER_OK;
}

int sscater_delta_update(const sscater_delta_spec* spec, const sscater_delta_memory* memory,
                         const sscater_token_rows* rows, const float* initial, const void* q, const void* k,
                         const void* v, const void* a, const void* b, const float* rate, const float* bias, void* out,
                         void* workspace, size_t workspace_bytes, void* stream) {
    if (!delta_ok(spec, memory, rows) || (uintptr_t)initial % 16) return SSCATER_E_INVALID_ARG;
    if ((rate == nullptr) != (bias == nullptr) || (uintptr_t)rate % 4 || (uintptr_t)bias % 4) return SSCATER_E_INVALID_ARG;
    const int size = memory->dtype == SSCATER_F32 ? 4 : 2;
    if (rows->tokens > 0) {
        for (const void* p : {q, k, v, a, b})
            if (!p || (uintptr_t)p % size) return SSCATER_E_INVALID_ARG;
        if (!out || (uintptr_t)out % 16) return SSCATER_E_INVALID_ARG;
    } else if (!initial || initial == memory->state) {
        return SSCATER_OK;
    }
    DeltaArgs x;
    x.rows.tokens = rows->tokens; x.rows.max_new = rows->max_new; x.rows.batch = memory->batch;
    x.rows.start = rows->tokens ? rows->start : nullptr; x.rows.past = nullptr;
    x.from = initial ? initial : memory->state;
    x.state = memory->state;
    x.q = q; x.k = k; x.v = v; x.a = a; x.b = b; x.rate = rate; x.bias = bias; x.out = out;
    x.ldq = spec->q_stride; x.ldk = spec->k_stride; x.ldv = spec->v_stride; x.lda = spec->a_stride; x.ldb = spec->b_stride;
    x.heads = memory->heads; x.group = memory->heads / memory->qk_heads;
    x.unit = spec->unit; x.eps = spec->eps; x.scale = spec->scale; x.item0 = 0;
    if (size == 4) launch_delta<true>(x, memory->key_dim, memory->value_dim, (hipStream_t)stream);
    else launch_delta<false>(x, memory->key_dim, memory->value_dim, (hipStream_t)stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSCATER_OK : report_hip_error(e);
}

}  // extern "C"
