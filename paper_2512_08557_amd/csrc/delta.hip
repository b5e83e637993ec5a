// The gated delta rule: a memory of fixed size for every stream and head, a matrix
// S [key_dim][value_dim] in fp32 that is read and corrected by every token:
//
//   u = beta (v - alpha S^T k),  S = alpha S + k u^T,  o = scale S^T q
//
// Tokens one by one: a wavefront owns 32 columns of a head's state in its registers
// (columns do not depend on one another).  Lane 8 c + r holds the r-th eighth of the
// rows of columns 4 c .. 4 c + 3, so a product with the state is key_dim / 2
// multiplications a lane and a sum between eight neighbouring lanes, and q and k come
// as one run of values for each lane.  alpha and beta are formed for 64 tokens at a time,
// a token a lane.  Bound by the states' way through memory where every stream brings a
// token (3348 streams of 8 heads of 32 x 32: 39 us, 5.6 TB/s), else by a token's chain
// of products and sums, 0.7 us.
//
// Stretches of 64 tokens at once: with G the running sum of log(alpha) within one, the
// corrections u are the solution of a triangular system that no state is in,
//
//   (I + A) U = X,  A_ij = beta_i e^(G_i - G_j) k_i . k_j (j < i),  X = beta (V - e^G K S)
//   O = scale (e^G Q S + P U),  P_ij = e^(G_i - G_j) q_i . k_j (j <= i)
//   S <- e^G_63 S + (e^(G_63 - G) K)^T U
//
// so T = (I + A)^-1 and P are formed for all stretches at once (chunk_kernel), and what is
// left from one to the next is five matrix products (state_kernel), each workgroup with 16
// columns of a state.  Those with T and P are products in the fp32 instructions; those with
// keys, queries and the state go through the bf16 ones, sixteen times as fast, with an fp32
// value cut into three bf16 planes that hold its 24 bits, and of the planes' products those
// that an fp32 sum holds: three with bf16 keys, six with fp32 ones.  A 16 x 16 result has its rows 4 g ..
// 4 g + 3 in lane 16 g + column, which is also where the next product wants its second
// operand's rows if the first's columns come in the same order, so S, X and U pass from
// product to product as they stand, between wavefronts through LDS.  Exponents are
// differences of sums in 64 bits: e^G_j may be zero where e^(G_i - G_j) is not.
#include "tokens.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

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
    int parts, length;     // of a stream, and the stretches of one
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

// Values as they lie in memory, made fp32 where they are used: a conversion beside the load would wait for it there.
template <bool F32>
struct Raw4 {
    uint32_t w[F32 ? 4 : 2];
    __device__ __forceinline__ void load(const void* p, int64_t i) {
        __builtin_memcpy(w, (const char*)p + i * (F32 ? 4 : 2), sizeof w);
    }
    __device__ __forceinline__ f4v get() const {
        if constexpr (F32) return f4v{__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3])};
        else return f4v{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xFFFF0000u), __uint_as_float(w[1] << 16),
                        __uint_as_float(w[1] & 0xFFFF0000u)};
    }
};
template <bool F32>
struct Raw1 {
    typename std::conditional<F32, uint32_t, uint16_t>::type w;
    __device__ __forceinline__ void load(const void* p, int64_t i) { w = ((const decltype(w)*)p)[i]; }
    __device__ __forceinline__ float get() const { return __uint_as_float(F32 ? (uint32_t)w : (uint32_t)w << 16); }
};

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
        float q[R], k[R], v[4];
    };
    auto fetch = [&](int64_t t) __attribute__((always_inline)) {
        Token x;
        values_at<F32>(a.q, t * a.ldq + hk * DK + r0, x.q);
        values_at<F32>(a.k, t * a.ldk + hk * DK + r0, x.k);
        values_at<F32>(a.v, t * a.ldv + h * DV + c0, x.v);
        return x;
    };
    Token next;
    if (n > 0) next = fetch(first);
    float alphas = 0.f, betas = 0.f;
    for (int i = 0; i < n; ++i) {
        const int64_t t = first + i;
        if (i % 64 == 0) {
            const int64_t mine = t + min(lane, n - 1 - i);
            alphas = expf(log_alpha(value_at<F32>(a.a, mine * a.lda + h), rate, bias, raw));
            betas = beta_of(value_at<F32>(a.b, mine * a.ldb + h), raw);
        }
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
            fq *= __builtin_amdgcn_rsqf(sum8(qq) + a.eps);
            fk = __builtin_amdgcn_rsqf(sum8(kk) + a.eps);
        }
        const float alpha = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(alphas), i % 64)),
                    beta = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(betas), i % 64));
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

// ---- stretches of tokens ----------------------------------------------------

constexpr int CHUNK = 64;
// What is kept of a stretch for each head: the ten lower tiles of T and of P, each as a wavefront reads it as a first
// operand (lane 16 g + r: row r, columns 4 g .. 4 g + 3), four factors of every token, e^G_63 and whether something is
// infinite, NaN or, in T, so large that U might be.
constexpr int MATS_P = 10 * 256, MATS_TOKEN = 20 * 256, MATS_LAST = MATS_TOKEN + 4 * CHUNK, MATS = MATS_LAST + 16;
enum { TOKEN_K, TOKEN_U, TOKEN_Q, TOKEN_BETA };

__device__ __forceinline__ int lower(int i, int j) { return i * (i + 1) / 2 + j; }

__device__ __forceinline__ f4v mfma4(float x, float y, f4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(x, y, c, 0, 0, 0);
}

// A product of 16 x 16 tiles.
__device__ __forceinline__ f4v tile_product(const f4v x, const f4v y, f4v c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = mfma4(x[e], y[e], c);
    return c;
}

// The stretch that workgroup `slot` of a call has: a sequence's are first / CHUNK + b onwards, as many as it needs at most.
__device__ __forceinline__ int slot_of(int first, int b) { return first / CHUNK + b; }

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u; }
// Of 2^e or more, infinite or NaN.
__device__ __forceinline__ bool beyond(float v, int e) { return (__float_as_uint(v) & 0x7F800000u) >= (uint32_t)(127 + e) << 23; }
// T and X below these make 64 sums that are finite.
constexpr int T_LIMIT = 20, X_LIMIT = 100;
constexpr int MAX_FLAGS = 32;                          // of a part: see state_kernel

// A workgroup a stretch and head: scores of keys and queries (bf16 in bf16 instructions: exact products), T by
// substitution in the diagonal tiles and products below them.  (12312 stretches of fp32 heads of 64: 215 us for 265 MB
// written and twice that read; matrix cores 30 % busy.)
template <bool F32, int DK>
__global__ __launch_bounds__(256) void chunk_kernel(DeltaArgs a, float* mats) {
    constexpr int NF = F32 ? DK / 16 : DK / 32;        // 16-byte pieces of a row that a lane holds
    constexpr int TILE = 16 * 20;                      // 16 rows of 16 values, 20 apart: rows on different banks
    __shared__ __attribute__((aligned(16))) float amat[10 * TILE], pmat[10 * TILE];
    // keys as operands, then T
    __shared__ __attribute__((aligned(16))) float shared[(4 * NF * 256 > 10 * TILE ? 4 * NF * 256 : 10 * TILE)];
    __shared__ double total[CHUNK];
    __shared__ float beta[CHUNK], unit_k[CHUNK], unit_q[CHUNK];
    __shared__ int bad[4];
    const int64_t id = a.item0 + blockIdx.x;
    const int h = (int)(id % a.heads), slot = (int)(id / a.heads);
    int lo = 0, hi = a.rows.batch - 1;
    int first, n;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        rows_of(a.rows, mid, first, n);
        if (slot_of(first, mid) <= slot) lo = mid; else hi = mid - 1;
    }
    rows_of(a.rows, lo, first, n);
    const int c = slot - slot_of(first, lo);
    if (c < 0 || c >= (n + CHUNK - 1) / CHUNK) return;
    const int m = min(CHUNK, n - c * CHUNK);
    const int64_t t0 = first + c * CHUNK;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int wq = 3 - w, hk = h / a.group;            // its row tile of Q: as many tiles of P as the others have of A
    bool odd = false;
    // rows 16 w + r of K and 16 wq + r of Q
    uint4 kf[NF], qf[NF];
    {
        const int tk = 16 * w + r, tq = 16 * wq + r;
        constexpr int E = F32 ? 4 : 8;
        const char* pk = (const char*)a.k + ((t0 + min(tk, m - 1)) * a.ldk + hk * DK) * (F32 ? 4 : 2) + g * 16;
        const char* pq = (const char*)a.q + ((t0 + min(tq, m - 1)) * a.ldq + hk * DK) * (F32 ? 4 : 2) + g * 16;
        float kk = 0.f, qq = 0.f;
#pragma unroll
        for (int t = 0; t < NF; ++t) {
            __builtin_memcpy(&kf[t], pk + t * 64, 16);
            __builtin_memcpy(&qf[t], pq + t * 64, 16);
            if (tk >= m) kf[t] = make_uint4(0, 0, 0, 0);
            if (tq >= m) qf[t] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int t = 0; t < NF; ++t) {
            const uint32_t ku[4] = {kf[t].x, kf[t].y, kf[t].z, kf[t].w}, qu[4] = {qf[t].x, qf[t].y, qf[t].z, qf[t].w};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float kv = __uint_as_float(F32 ? ku[e & 3] : e & 1 ? ku[e / 2] & 0xFFFF0000u : ku[e / 2] << 16);
                const float qv = __uint_as_float(F32 ? qu[e & 3] : e & 1 ? qu[e / 2] & 0xFFFF0000u : qu[e / 2] << 16);
                // (an infinite query has the state's sign, which a sum over the stretch's tokens would lose)
                odd |= !finite(kv) || (!a.unit && fabsf(qv) == INFINITY);
                kk = fmaf(kv, kv, kk);
                qq = fmaf(qv, qv, qq);
            }
            *(uint4*)&shared[((w * NF + t) * 64 + lane) * 4] = kf[t];
        }
        kk += __shfl_xor(kk, 16);
        qq += __shfl_xor(qq, 16);
        kk += __shfl_xor(kk, 32);
        qq += __shfl_xor(qq, 32);
        if (g == 0) {
            // (behind the last token zero, whatever eps)
            unit_k[tk] = tk >= m ? 0.f : a.unit ? 1.f / sqrtf(kk + a.eps) : 1.f;
            unit_q[tq] = tq >= m ? 0.f : (a.unit ? 1.f / sqrtf(qq + a.eps) : 1.f) * a.scale;
        }
    }
    if (w == 0) {
        const bool raw = a.rate != nullptr, live = lane < m;
        const int64_t t = t0 + min(lane, m - 1);
        const float la = log_alpha(value_at<F32>(a.a, t * a.lda + h), raw ? a.rate[h] : 0.f, raw ? a.bias[h] : 0.f, raw);
        const float be = beta_of(value_at<F32>(a.b, t * a.ldb + h), raw);
        odd |= live && !(finite(la) && finite(be));
        double sum = live ? la : 0.;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const double v = __shfl_up(sum, o);
            if (lane >= o) sum += v;
        }
        total[lane] = sum;
        beta[lane] = live ? be : 0.f;
    }
    odd = __ballot(odd) != 0;
    if (lane == 0) bad[w] = odd;
    __syncthreads();
    auto dot = [&](const uint4 (&x)[NF], int j) __attribute__((always_inline)) {
        f4v c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < NF; ++t) {
            const uint4 y = *(const uint4*)&shared[((j * NF + t) * 64 + lane) * 4];
            if constexpr (F32) {
                const uint32_t u[4] = {x[t].x, x[t].y, x[t].z, x[t].w}, v[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) c = mfma4(__uint_as_float(u[e]), __uint_as_float(v[e]), c);
            } else {
                c = mfma_bf16(x[t], y, c);
            }
        }
        return c;
    };
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const double gj = total[16 * j + r];
        const float kj = unit_k[16 * j + r];
        if (j <= w) {
            const f4v d = dot(kf, j);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = 16 * w + 4 * g + e;
                const float f = beta[i] * unit_k[i] * kj * expf((float)(total[i] - gj));
                amat[lower(w, j) * TILE + (4 * g + e) * 20 + r] = 16 * j + r < i ? f * d[e] : 0.f;
            }
        }
        if (j <= wq) {
            const f4v d = dot(qf, j);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = 16 * wq + 4 * g + e;
                const float f = unit_q[i] * kj * expf((float)(total[i] - gj));
                pmat[lower(wq, j) * TILE + (4 * g + e) * 20 + r] = 16 * j + r <= i ? f * d[e] : 0.f;
            }
        }
    }
    __syncthreads();
    float* const out = mats + id * MATS;
    // T's diagonal tile w by substitution, a column a lane (four times the same)
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        x[i] = i == r ? 1.f : 0.f;
#pragma unroll
        for (int k4 = 0; k4 < (i + 3) / 4; ++k4) {
            const f4v v = *(const f4v*)&amat[lower(w, w) * TILE + i * 20 + 4 * k4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (4 * k4 + e < i) x[i] = fmaf(-v[e], x[4 * k4 + e], x[i]);
        }
    }
    f4v column[4];                                     // T's tiles (i, w), i >= w
    f4v diag;
#pragma unroll
    for (int e = 0; e < 4; ++e) diag[e] = g == 0 ? x[e] : g == 1 ? x[4 + e] : g == 2 ? x[8 + e] : x[12 + e];
    auto keep = [&](int i, const f4v v) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) shared[lower(i, w) * TILE + (4 * g + e) * 20 + r] = v[e];
    };
    auto operand = [&](const float* from, int tile) __attribute__((always_inline)) {
        return *(const f4v*)&from[tile * TILE + r * 20 + 4 * g];
    };
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i == w) {
            column[i] = diag;
            keep(i, diag);
        }
    __syncthreads();
#pragma unroll
    for (int i = 1; i < 4; ++i)
        if (i > w) {
            f4v y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < i; ++k)
                if (k >= w) y = tile_product(operand(amat, lower(i, k)), column[k], y);
            y = tile_product(operand(shared, lower(i, i)), y, f4v{0.f, 0.f, 0.f, 0.f});
            column[i] = -y;
            keep(i, column[i]);
        }
    bool large = false;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i >= w)
#pragma unroll
            for (int e = 0; e < 4; ++e) large |= beyond(column[i][e], T_LIMIT);
    large = __ballot(large) != 0;
    if (lane == 0 && large) bad[w] = 1;
    __syncthreads();
    for (int t = w; t < 10; t += 4) {
        *(f4v*)&out[t * 256 + lane * 4] = operand(shared, t);
        *(f4v*)&out[MATS_P + t * 256 + lane * 4] = operand(pmat, t);
    }
    if (w == 0) {
        const float since = expf((float)total[lane]), left = expf((float)(total[CHUNK - 1] - total[lane]));
        out[MATS_TOKEN + TOKEN_K * CHUNK + lane] = beta[lane] * since * unit_k[lane];
        out[MATS_TOKEN + TOKEN_U * CHUNK + lane] = left * unit_k[lane];
        out[MATS_TOKEN + TOKEN_Q * CHUNK + lane] = since * unit_q[lane];
        out[MATS_TOKEN + TOKEN_BETA * CHUNK + lane] = beta[lane];
        if (lane == CHUNK - 1) out[MATS_LAST] = since;
        if (lane == 0) out[MATS_LAST + 1] = bad[0] | bad[1] | bad[2] | bad[3] ? 1.f : 0.f;
    }
}

// From one stretch to the next.  A workgroup has 16 columns of a head's state; wavefronts 0 to 3 take it through the
// stretches (X, then U, then S), 4 to 7 form the outputs beside them, so that a SIMD's two wavefronts fill each other's
// waits.  An operand of the next stretch is loaded into its registers as soon as this one's product has taken them; every
// load is made whatever the stretch, so that the number under way is known where they are waited for.
//
// Where streams and heads leave compute units idle, a stream is cut into a.parts of a.length stretches.  A part takes S
// to M S + B, so a first launch (OUT = false) takes zeros (the first part: the state, and puts it aside too) and, in more
// columns, the unit matrix through all parts but the last, without outputs, and the workgroups of the second begin with
// the product of the parts before theirs.
//
// Bound by the way through a stretch: three products and meetings after one another, 2.1 us (523 stretches, four streams,
// 8 fp32 heads of 64 x 128: 1120 us with 256 workgroups, with fp32 products throughout a tenth more; 3348 tokens of 8 bf16
// heads of 64 x 64 in eight parts: 20 and 22, 23 and 26).  Keys and queries are cut while the chain is at its first product; in
// the second's time, cutting was 70 us more.  Matrices that come from memory later than a stretch after their loads are 70
// us of it; touching them three stretches ahead, by the outputs' wavefronts or by a ninth, gave none of that back.
template <bool F32, int DK, int DV, bool OUT>
__global__ __launch_bounds__(OUT ? 512 : 256) void state_kernel(DeltaArgs a, const float* mats, float* parts) {
    constexpr int S = F32 ? 4 : 2;
    constexpr int NT = DK / 16, OWN = (NT + 3) / 4;    // row tiles of the state, and those of a wavefront
    __shared__ __attribute__((aligned(16))) f4v sbuf[NT][64], zbuf[NT][64], xbuf[4][64], ubuf[4][64], ybuf[4][64];
    // PL: the state and Y as three bf16 planes each, second operands of 32 rows (two tiles), and as first ones the keys, one
    // plane if they are bf16 and three if not.  Without outputs fp32 keys stay fp32: nobody is there to cut them.
    constexpr bool PL = !F32 || OUT;
    constexpr int KP = F32 ? 3 : 1;
    __shared__ __attribute__((aligned(16))) uint4 splanes[PL ? NT / 2 * 3 : 1][64], yplanes[PL ? 2 * 3 : 1][64];
    // The stretch's keys and, from the outputs' wavefronts, the next one's.  PL: 32 columns' 16-byte pieces are four of
    // columns 4 g .. 4 g + 3 and of 4 g + 16 .. 4 g + 19, as the products take them.
    constexpr int PITCH = DK * (PL ? 2 : 4) + 16, PLANE = CHUNK * PITCH, KEYS = (PL ? KP : 1) * PLANE;
    __shared__ __attribute__((aligned(16))) char kbuf[(OUT ? 2 : 1) * KEYS];
    __shared__ float part[2][16][16];
    __shared__ uint32_t bad[4];
    // the columns of a head follow one another on one XCD (workgroup id mod 8), whose L2 then has its keys and matrices
    constexpr int BLOCKS = (OUT ? DV : DV + DK) / 16;
    const int64_t id = a.item0 + blockIdx.x, of = id / 8 / BLOCKS;
    const int64_t which = of / (OUT ? a.parts : a.parts - 1) * 8 + id % 8;
    const int seg = (int)(of % (OUT ? a.parts : a.parts - 1)), block = (int)(id / 8 % BLOCKS);
    if (which >= (int64_t)a.rows.batch * a.heads) return;
    const int b = (int)(which / a.heads), h = (int)(which % a.heads), hk = h / a.group;
    int first, n;
    rows_of(a.rows, b, first, n);
    const bool unit = !OUT && block >= DV / 16;        // columns of the unit matrix
    const int all = (n + CHUNK - 1) / CHUNK, c0 = min(all, seg * a.length), chunks = min(all, c0 + a.length);
    if (OUT && n == 0 && a.from == a.state) return;
    if (seg > 0 ? c0 == all : unit) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int w = wave & 3, wq = 3 - w, col = (block - (unit ? DV / 16 : 0)) * 16 + r;
    // a part's M, as first operands, B, as results, and whether M has large values, infinities or NaN (of the wavefronts that
    // formed it)
    constexpr int PART_FLAGS = DK * DK + DK * DV, FLAGS = DK / 16 * 4, PART = PART_FLAGS + MAX_FLAGS;
    float* const part0 = parts + which * a.parts * PART;
    // A product with such an M may be infinite or NaN where the tokens one after the other are not (a large key before which
    // the memory is empty): the stretches of all parts before are gone through here, too.
    bool whole = false;
    if constexpr (OUT) {
        for (int i = lane; i < (seg - 1) * FLAGS; i += 64) whole |= part0[(1 + i / FLAGS) * PART + PART_FLAGS + i % FLAGS] != 0.f;
        whole = __ballot(whole) != 0;
    }
    const int cb = whole ? 0 : c0, joins = whole ? 1 : seg;
    auto b_of = [&](int j, int tile) __attribute__((always_inline)) {
        return (f4v*)(part0 + j * PART + DK * DK + ((int64_t)tile * (DV / 16) + block) * 256 + lane * 4);
    };
    // of the stretch whose operands are loaded next, moved on from one to the next: a stretch's worth of scalar
    // multiplications is time on every wavefront's way
    const int64_t row0 = first + (int64_t)cb * CHUNK, step_m = (int64_t)a.heads * MATS;
    const float* mx = mats + ((int64_t)(slot_of(first, b) + cb) * a.heads + h) * MATS;
    const float *mu = mx, *ms = mx;
    const uint32_t ldk = (uint32_t)a.ldk * S, ldq = (uint32_t)a.ldq * S, ldv = (uint32_t)a.ldv * S;
    auto tokens = [&](int c) __attribute__((always_inline)) { return min(CHUNK, n - c * CHUNK); };
    auto put = [&](int64_t t, float v) __attribute__((always_inline)) {
        const int64_t to = (t * a.heads + h) * DV + col;
        if constexpr (F32) ((float*)a.out)[to] = v;
        else ((uint16_t*)a.out)[to] = (uint16_t)bf16_pair(v, v);
    };
    typedef uint32_t u2v __attribute__((ext_vector_type(2)));
    auto planes_of = [&](const f4v v, u2v (&x)[3]) __attribute__((always_inline)) {
        uint32_t a[3], b[3];
        cut_pair(__float_as_uint(v[0]), __float_as_uint(v[1]), a[0], a[1], a[2]);
        cut_pair(__float_as_uint(v[2]), __float_as_uint(v[3]), b[0], b[1], b[2]);
#pragma unroll
        for (int i = 0; i < 3; ++i) x[i] = u2v{a[i], b[i]};
    };
    // a tile as planes, behind or before its neighbour's rows
    auto cut = [&](const f4v v, uint4 (*to)[64], int tile) __attribute__((always_inline)) {
        u2v x[3];
        planes_of(v, x);
#pragma unroll
        for (int i = 0; i < 3; ++i) *(u2v*)((char*)&to[tile / 2 * 3 + i][lane] + tile % 2 * 8) = x[i];
    };
    // 32 rows' product: of nine of planes the six that fp32 holds
    auto plane_products = [&](const uint4 (&x)[KP], const uint4 (*y)[64], f4v (&c)[3]) __attribute__((always_inline)) {
        const uint4 y0 = y[0][lane], y1 = y[1][lane], y2 = y[2][lane];
        c[0] = mfma_bf16(x[0], y0, c[0]);
        c[1] = mfma_bf16(x[0], y1, c[1]);
        c[2] = mfma_bf16(x[0], y2, c[2]);
        if constexpr (KP == 3) {
            c[1] = mfma_bf16(x[1], y0, c[1]);
            c[2] = mfma_bf16(x[1], y1, c[2]);
            c[2] = mfma_bf16(x[2], y0, c[2]);
        }
    };
    // 16 rows of keys or queries, as operands of the product with the state, and that
    struct Rows {
        uint4 v[PL ? NT / 2 : NT][PL ? KP : 1];
    };
    auto operands = [&](const Raw4<F32> (&x)[NT]) __attribute__((always_inline)) {
        Rows rows;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if constexpr (!PL) {
                rows.v[t][0] = make_uint4(x[t].w[0], x[t].w[1], x[t].w[2], x[t].w[3]);
            } else if constexpr (F32) {
                u2v v[3];
                planes_of(x[t].get(), v);
#pragma unroll
                for (int i = 0; i < KP; ++i) {
                    uint4& u = rows.v[t / 2][i];
                    (t & 1 ? u.z : u.x) = v[i][0];
                    (t & 1 ? u.w : u.y) = v[i][1];
                }
            } else {
                uint4& u = rows.v[t / 2][0];
                (t & 1 ? u.z : u.x) = x[t].w[0];
                (t & 1 ? u.w : u.y) = x[t].w[1];
            }
        }
        return rows;
    };
    auto rows_times_state = [&](const Rows& x) __attribute__((always_inline)) {
        if constexpr (!PL) {
            // two sums: an instruction need not wait for the one before it
            f4v c[2] = {};
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                f4v v;
                __builtin_memcpy(&v, &x.v[t][0], 16);
                c[t & 1] = tile_product(v, sbuf[t][lane], c[t & 1]);
            }
            return c[0] + c[1];
        } else {
            f4v c[3] = {};
#pragma unroll
            for (int t = 0; t < NT / 2; ++t) plane_products(x.v[t], splanes + t * 3, c);
            return c[0] + (c[1] + c[2]);
        }
    };
    // 16 rows of keys into LDS, and as they lie there times the state
    auto keep_keys = [&](const Raw4<F32> (&x)[NT], int tile, char* to) __attribute__((always_inline)) {
        to += (16 * tile + r) * PITCH + 16 * g;
        const Rows rows = operands(x);
#pragma unroll
        for (int t = 0; t < (PL ? NT / 2 : NT); ++t)
#pragma unroll
            for (int i = 0; i < (PL ? KP : 1); ++i) *(uint4*)(to + i * PLANE + 64 * t) = rows.v[t][i];
    };
    auto keys_times_state = [&](int tile, const char* from) __attribute__((always_inline)) {
        f4v c[3] = {};
#pragma unroll
        for (int t = 0; t < NT / 2; ++t) {
            uint4 v[KP];
#pragma unroll
            for (int i = 0; i < KP; ++i) v[i] = *(const uint4*)(from + i * PLANE + (16 * tile + r) * PITCH + 64 * t + 16 * g);
            plane_products(v, splanes + t * 3, c);
        }
        return c[0] + (c[1] + c[2]);
    };
    // the same from all of a workgroup's wavefronts
    auto bad_columns = [&]() __attribute__((always_inline)) {
        return __builtin_amdgcn_readfirstlane((bad[0] | bad[1] | bad[2] | bad[3]) & 0xFFFFu);
    };
    const int sums = a.unit ? 4 : 2;                   // of a token taken by itself
    constexpr int HAND = PL ? 1 : 0;                   // meeting before those, for the state in fp32

    if (OUT && wave >= 4) {
        Raw4<F32> q[NT];
        f4v p[4], fq;
        uint32_t off = (uint32_t)(16 * wq + r) * ldq + 4 * g * S;
        const char* at = (const char*)a.q + (row0 * a.ldq + hk * DK) * S;
        const int64_t step_q = (int64_t)CHUNK * ldq;
        auto load_q = [&](int c) __attribute__((always_inline)) {
            const int m = tokens(c);
            if (m < CHUNK) off = (uint32_t)min(16 * wq + r, m - 1) * ldq + 4 * g * S;
#pragma unroll
            for (int t = 0; t < NT; ++t) q[t].load(at + off + 16 * t * S, 0);
            fq = *(const f4v*)&mx[MATS_TOKEN + TOKEN_Q * CHUNK + 16 * wq + 4 * g];
        };
        const uint32_t off_p = (MATS_P + lower(wq, 0) * 256 + lane * 4) * 4;
        auto load_p = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = *(const f4v*)((const char*)mu + off_p + (uint32_t)min(i, wq) * 1024);
        };
        // and the next stretch's keys, loaded a stretch before they are cut
        Raw4<F32> k[NT];
        const char* from = (const char*)a.k + (row0 * a.ldk + hk * DK) * S;
        const int64_t step_k = (int64_t)CHUNK * ldk;
        auto load_k = [&](int c) __attribute__((always_inline)) {
            const uint32_t off = (uint32_t)min(16 * w + r, tokens(c) - 1) * ldk + 4 * g * S;
#pragma unroll
            for (int t = 0; t < NT; ++t) k[t].load(from + off + 16 * t * S, 0);
        };
        if (chunks > cb) {
            load_k(cb);
            load_q(cb);
            load_p();
            keep_keys(k, w, kbuf + (cb & 1) * KEYS);
            if (cb + 1 < chunks) from += step_k;
            load_k(min(cb + 1, chunks - 1));
        }
        const int64_t out_row = (int64_t)a.heads * DV;
        char* to = (char*)a.out + ((row0 + 16 * wq + 4 * g) * out_row + h * DV + col) * S;
        lds_barrier();
        for (int j = 1; j < joins; ++j) {
            lds_barrier();
            lds_barrier();
        }
#pragma unroll 1
        for (int c = cb; c < chunks; ++c) {
            const int m = tokens(c), next = min(c + 1, chunks - 1);
            // beside the chain's first product
            const Rows queries = operands(q);
            keep_keys(k, w, kbuf + ((c + 1) & 1) * KEYS);
            if (c + 2 < chunks) from += step_k;
            load_k(min(c + 2, chunks - 1));
            lds_barrier();
            const uint32_t columns = bad_columns();
            if (columns)
                for (int i = m * sums + HAND; i > 0; --i) lds_barrier();
            f4v o[2] = {rows_times_state(queries), {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int e = 0; e < 4; ++e) o[0][e] *= fq[e];
            if (c + 1 < chunks) {
                at += step_q;
                mx += step_m;
            }
            load_q(next);
            lds_barrier();
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (t <= wq) o[t & 1] = tile_product(p[t], ubuf[t][lane], o[t & 1]);
            if (c + 1 < chunks) mu += step_m;
            load_p();
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = o[0][e] + o[1][e];
                char* const at = to + e * out_row * S;
                if (16 * wq + 4 * g + e < m && !(columns >> r & 1) && c >= c0) {
                    if constexpr (F32) *(float*)at = v;
                    else *(uint16_t*)at = (uint16_t)bf16_pair(v, v);
                }
            }
            to += CHUNK * out_row * S;
            lds_barrier();
        }
        return;
    }

    f4v s[OWN];
    // for the products with it; and as it is, which a slow stretch and the parts before take
    auto give = [&](int t, const f4v v) __attribute__((always_inline)) {
        if constexpr (PL) cut(v, splanes, t);
        else sbuf[t][lane] = v;
    };
    auto tile = [&](int o) __attribute__((always_inline)) { return NT < 4 ? min(w, NT - 1) : w + 4 * o; };
    const bool own = NT >= 4 || w < NT;
    auto state_at = [&](int o, int e) __attribute__((always_inline)) {
        return (which * DK + 16 * tile(o) + 4 * g + e) * DV + col;
    };
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
        if (OUT && a.parts > 1) {
            // the state put aside, or the first part's end
            s[o] = *b_of(seg == 0 || whole ? a.parts - 1 : 0, tile(o));
        } else if (seg == 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[o][e] = a.from[state_at(o, e)];
            if (!OUT && own) *b_of(a.parts - 1, tile(o)) = s[o];
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[o][e] = unit && 16 * tile(o) + 4 * g + e == col ? 1.f : 0.f;
        }
        if (own) sbuf[tile(o)][lane] = s[o];
        if (PL && own) cut(s[o], splanes, tile(o));
    }
    Raw4<F32> k[NT];
    Raw1<F32> v[4];
    f4v inv[4], fk, fb, fu;
    float last, keys_odd;
    uint32_t off_k = (uint32_t)(16 * w + r) * ldk + 4 * g * S, off_v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) off_v[e] = (uint32_t)(16 * w + 4 * g + e) * ldv + col * S;
    const char* keys = (const char*)a.k + (row0 * a.ldk + hk * DK) * S;
    const char* values = (const char*)a.v + (row0 * a.ldv + h * DV) * S;
    const int64_t step_k = (int64_t)CHUNK * ldk, step_v = (int64_t)CHUNK * ldv;
    // (the rows behind a stream's last token are that token once more)
    auto load_x = [&](int c) __attribute__((always_inline)) {
        const int m = tokens(c);
        if (m < CHUNK) {
            off_k = (uint32_t)min(16 * w + r, m - 1) * ldk + 4 * g * S;
#pragma unroll
            for (int e = 0; e < 4; ++e) off_v[e] = (uint32_t)min(16 * w + 4 * g + e, m - 1) * ldv + col * S;
        }
        if constexpr (!OUT)
#pragma unroll
            for (int t = 0; t < NT; ++t) k[t].load(keys + off_k + 16 * t * S, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e].load(values + off_v[e], 0);
        fk = *(const f4v*)&mx[MATS_TOKEN + TOKEN_K * CHUNK + 16 * w + 4 * g];
        fb = *(const f4v*)&mx[MATS_TOKEN + TOKEN_BETA * CHUNK + 16 * w + 4 * g];
        keys_odd = mx[MATS_LAST + 1];
    };
    const uint32_t off_m = (lower(w, 0) * 256 + lane * 4) * 4;
    auto load_u = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) inv[i] = *(const f4v*)((const char*)mu + off_m + (uint32_t)min(i, w) * 1024);
    };
    auto load_s = [&]() __attribute__((always_inline)) {
        fu = *(const f4v*)&ms[MATS_TOKEN + TOKEN_U * CHUNK + 16 * w + 4 * g];
        last = ms[MATS_LAST];
    };
    // Tokens one by one, for columns with infinities or NaN in a stretch, or values that might become some (all of them, if
    // in its keys or gates): a product with a triangle's zeros would carry them to the tokens before.  Thread 16 p + column has the p-th sixteenth of a
    // column's rows; the state after goes to zbuf.
    auto slowly = [&](int c, uint32_t columns) __attribute__((always_inline)) {
        constexpr int R = DK / 16;
        int none = 0;
        asm volatile("" : "+v"(none));                 // what follows is not worth registers of the loop around it
        const int p = (threadIdx.x >> 4) + none, r = (lane & 15) + none, column = col + none, m = tokens(c);
        const bool raw = a.rate != nullptr;
        const float rate = raw ? a.rate[h] : 0.f, bias = raw ? a.bias[h] : 0.f;
        float z[R];
        if constexpr (PL) {
#pragma unroll
            for (int o = 0; o < OWN; ++o)
                if (own) sbuf[tile(o)][lane] = s[o];
            lds_barrier();
        }
        auto place = [&](f4v (&buf)[NT][64], int i) __attribute__((always_inline)) {
            const int row = p * R + i;
            return &((float*)&buf[row / 16][16 * (row % 16 / 4) + r])[row % 4];
        };
#pragma unroll
        for (int i = 0; i < R; ++i) z[i] = *place(sbuf, i);
        auto sum = [&](float v, int turn) __attribute__((always_inline)) {
            part[turn][p][r] = v;
            lds_barrier();                             // as many as the other wavefronts wait for: `sums` a token
            v = 0.f;
            for (int i = 0; i < 16; ++i) v += part[turn][i][r];
            return v;
        };
        for (int i = 0; i < m; ++i) {
            const int64_t t = first + (int64_t)c * CHUNK + i;
            float kk = 0.f, qq = 0.f, k[R], q[R];
            values_at<F32>(a.k, t * a.ldk + hk * DK + p * R, k);
            values_at<F32>(a.q, t * a.ldq + hk * DK + p * R, q);
#pragma unroll
            for (int j = 0; j < R; ++j) {
                kk = fmaf(k[j], k[j], kk);
                qq = fmaf(q[j], q[j], qq);
            }
            const float fk = a.unit ? 1.f / sqrtf(sum(kk, 0) + a.eps) : 1.f;
            const float fq = (a.unit ? 1.f / sqrtf(sum(qq, 1) + a.eps) : 1.f) * a.scale;
            const float alpha = expf(log_alpha(value_at<F32>(a.a, t * a.lda + h), rate, bias, raw));
            float dot = 0.f, o = 0.f;
#pragma unroll
            for (int j = 0; j < R; ++j) {
                k[j] *= fk;
                dot = fmaf(z[j], k[j], dot);
            }
            const float u = beta_of(value_at<F32>(a.b, t * a.ldb + h), raw) *
                            ((unit ? 0.f : value_at<F32>(a.v, t * a.ldv + h * DV + column)) - alpha * sum(dot, 0));
#pragma unroll
            for (int j = 0; j < R; ++j) {
                z[j] = fmaf(k[j], u, alpha * z[j]);
                o = fmaf(z[j], q[j], o);
            }
            o = sum(o, 1) * fq;
            if (OUT && p == 0 && (columns >> r & 1) && c >= c0) put(t, o);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) *place(zbuf, i) = z[i];
    };
    if (chunks > cb) {
        load_x(cb);
        load_u();
        load_s();
    }
    lds_barrier();
    if constexpr (OUT) {
#pragma unroll 1
        for (int j = 1; j < joins; ++j) {
            f4v y[OWN];
#pragma unroll
            for (int o = 0; o < OWN; ++o) {
                y[o] = *b_of(j, tile(o));
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    y[o] = tile_product(*(const f4v*)(part0 + j * PART + (tile(o) * NT + t) * 256 + lane * 4), sbuf[t][lane], y[o]);
            }
            lds_barrier();
#pragma unroll
            for (int o = 0; o < OWN; ++o) {
                s[o] = y[o];
                if (own) sbuf[tile(o)][lane] = s[o];
                if (PL && own) cut(s[o], splanes, tile(o));
            }
            lds_barrier();
        }
    }
#pragma unroll 1
    for (int c = cb; c < chunks; ++c) {
        const int m = tokens(c), next = min(c + 1, chunks - 1);
        char* const kb = kbuf + (OUT ? (c & 1) * KEYS : 0);
        f4v x;
        if constexpr (OUT) {
            x = keys_times_state(w, kb);
        } else {
            keep_keys(k, w, kb);
            x = rows_times_state(operands(k));
        }
        bool odd = keys_odd != 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float value = 16 * w + 4 * g + e < m && !unit ? v[e].get() : 0.f;
            x[e] = fmaf(fb[e], value, -fk[e] * x[e]);
            odd |= beyond(x[e], X_LIMIT);
        }
        xbuf[w][lane] = x;
        const uint64_t lanes = __ballot(odd);
        if (lane == 0) bad[w] = (uint32_t)(lanes | lanes >> 32) | (uint32_t)(lanes >> 16 | lanes >> 48);
        if (c + 1 < chunks) {
            keys += step_k;
            values += step_v;
            mx += step_m;
        }
        load_x(next);
        lds_barrier();
        // (read before the columns are known: a slow stretch leaves them)
        f4v xs[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) xs[t] = xbuf[t][lane];
        const uint32_t columns = bad_columns();
        if (columns) slowly(c, columns);
        f4v u[2] = {};
#pragma unroll
        for (int t = 0; t < 4; ++t)
            if (t <= w) u[t & 1] = tile_product(inv[t], xs[t], u[t & 1]);
        u[0] += u[1];
        if (OUT) ubuf[w][lane] = u[0];
#pragma unroll
        for (int e = 0; e < 4; ++e) u[0][e] *= fu[e];
        if constexpr (PL) cut(u[0], yplanes, w);
        else ybuf[w][lane] = u[0];
#pragma unroll
        for (int i = 0; i < OWN; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[i][e] *= last;
        if (c + 1 < chunks) mu += step_m;
        load_u();
        lds_barrier();
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            if constexpr (!PL) {
                f4v more = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    f4v key;
#pragma unroll
                    for (int e = 0; e < 4; ++e) key[e] = *(const float*)(kb + (16 * t + 4 * g + e) * PITCH + (16 * tile(i) + r) * 4);
                    if (t & 1) more = tile_product(key, ybuf[t][lane], more);
                    else s[i] = tile_product(key, ybuf[t][lane], s[i]);
                }
                s[i] += more;
            } else {
                // (a transposing read: 16 lanes take 4 rows of 16 keys' values, each lane a column of them)
                typedef short s4v __attribute__((ext_vector_type(4)));
                typedef __attribute__((address_space(3))) s4v lds_s4v;
                f4v sum[3] = {s[i]};
                const lds_char* at = (const lds_char*)kb + (4 * g + (r >> 2)) * PITCH + tile(i) / 2 * 64 + (r & 3) * 16 + tile(i) % 2 * 8;
#pragma unroll
                for (int t = 0; t < 4; t += 2) {
                    uint4 key[KP];
#pragma unroll
                    for (int p = 0; p < KP; ++p) {
                        const s4v k0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v*)(at + p * PLANE + 16 * t * PITCH));
                        const s4v k1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v*)(at + p * PLANE + 16 * (t + 1) * PITCH));
                        __builtin_memcpy(&key[p], &k0, 8);
                        __builtin_memcpy((char*)&key[p] + 8, &k1, 8);
                    }
                    plane_products(key, yplanes + t / 2 * 3, sum);
                }
                s[i] = sum[0] + (sum[1] + sum[2]);
            }
            if (columns >> r & 1) s[i] = zbuf[tile(i)][lane];
            if (own) give(tile(i), s[i]);
        }
        if (c + 1 < chunks) ms += step_m;
        load_s();
        lds_barrier();
    }
    if (!OUT && unit) {
        bool large = false;
#pragma unroll
        for (int o = 0; o < OWN; ++o)
#pragma unroll
            for (int e = 0; e < 4; ++e) large |= beyond(s[o][e], T_LIMIT);
        large = __ballot(large) != 0;
        if (lane == 0) part0[seg * PART + PART_FLAGS + col / 16 * 4 + w] = large ? 1.f : 0.f;
    }
    if (!own) return;
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
        if (OUT) {
            if (chunks < all) break;                   // a later part has the stream's end
#pragma unroll
            for (int e = 0; e < 4; ++e) a.state[state_at(o, e)] = s[o][e];
        } else if (!unit) {
            *b_of(seg, tile(o)) = s[o];
        } else {
            // column 4 x + y of a tile is lane 16 x + row's y-th value of the operand
#pragma unroll
            for (int e = 0; e < 4; ++e)
                part0[seg * PART + (tile(o) * NT + col / 16) * 256 + ((r / 4) * 16 + 4 * g + e) * 4 + r % 4] = s[o][e];
        }
    }
}

namespace {

constexpr int MAX_PARTS = 64;

// Stretches of a call, parts of a stream and the stretches of a part; no stretches: tokens one by one.
struct DeltaPlan {
    int64_t slots;
    int parts, length;
};

template <bool F32, int DK>
void launch_chunks(DeltaArgs a, int64_t slots, float* mats, hipStream_t s) {
    for (int64_t g = 0; g < slots * a.heads; g += LAUNCH_GROUPS) {
        a.item0 = g;
        chunk_kernel<F32, DK><<<dim3((unsigned)std::min(LAUNCH_GROUPS, slots * a.heads - g)), dim3(256), 0, s>>>(a, mats);
    }
}

// Tokens one by one or in stretches, and the parts of the streams: whichever takes least by what the pieces take, in
// microseconds.  A token is 0.35 and 0.0055 for each row of a head's state, or 0.45 for each thousand wavefronts where
// there are many; a stretch with its outputs 2.1 of bf16 and 2.9 of fp32 tokens (2.1 for a single round, more for many,
// whose operands are memory's time), without 2 (two workgroups on a compute unit), a product of parts 0.8; a launch of
// states 4 for each round over the card, chunk_kernel 1 for 150 heads' stretches, 80 of fp32; the further launches 5 each.
// (Heads of 64 x 64 in bf16, one by one and in stretches: 8 heads, 8 tokens 10.2 and 13.2, 16 tokens 16.0 and 13.2, 64
// tokens 49 and 14; 128 heads, 16 tokens 16.3 and 18.3, 32 tokens 27.6 and 18.8; 8000 heads, 64 tokens 462 and 715, 192
// tokens 1329 and 1288; 4000 heads in fp32, 192 tokens 651 and 848; 2400 heads of 32 x 32, 64 tokens 76 and 118.  Of 128 x
// 128 in bf16: 8 heads, 8 tokens 14.1 and 13.8, 16 tokens 22.7 and 14.1; 128 heads, 16 tokens 24.1 and 30.5, 32 tokens 40.6
// and 31.2; 2000 heads, 64 tokens 460 and 475, 192 tokens 1361 and 843; in fp32 8 heads, 8 tokens 13.5 and 17.1, 16 tokens
// 20.9 and 17.6; 128 heads, 32 tokens 37.0 and 37.7, 64 tokens 66.9 and 42.7; 2000 heads, 192 tokens 1250 and 1063.  The
// constants are the same for them, which is wrong only for thousands of heads and tokens enough: there they go one by one.)
DeltaPlan delta_plan(const sscater_delta_memory* m, const sscater_token_rows* r) {
    DeltaPlan p = {0, 1, 0};
    const bool f32 = m->dtype == SSCATER_F32;
    const double heads = (double)m->batch * m->heads, n = r->max_new, blocks = m->value_dim / 16;
    const double token = 5. + n * std::max(0.35 + 0.0055 * m->key_dim, 0.00045 * heads * blocks / 2.);
    const int64_t most = ((int64_t)r->max_new + CHUNK - 1) / CHUNK;
    double best = token;
    for (int64_t k = 1; k <= std::min(most, (int64_t)MAX_PARTS); ++k) {
        const int64_t length = (most + k - 1) / k;
        const double out = std::ceil(heads * blocks * k / 256.), in = std::ceil(heads * (blocks + m->key_dim / 16) * (k - 1) / 512.);
        if ((most + length - 1) / length != k || (k > 1 && out > 8.)) continue;
        const double cost = 8. + heads * most / (f32 ? 80. : 150.) + out * (4. + (f32 ? 2.9 : 2.1) * length) +
                            (k > 1 ? 5. + in * (4. + 2. * length) + 0.8 * (k - 2) : 0.);
        if (cost < best) {
            best = cost;
            p.slots = std::min((int64_t)r->tokens, (int64_t)r->max_new * m->batch) / CHUNK + m->batch;
            p.parts = (int)k;
            p.length = (int)length;
        }
    }
    return p;
}

size_t delta_bytes(const DeltaPlan& p, const sscater_delta_memory* m) {
    const size_t part = (size_t)m->key_dim * (m->key_dim + m->value_dim) + MAX_FLAGS;
    return 4 * m->heads * (p.slots * (size_t)MATS + (p.parts > 1 ? (size_t)m->batch * p.parts * part : 0));
}

template <bool F32, int DK, int DV, bool OUT>
void launch_states(DeltaArgs a, const float* mats, float* parts, hipStream_t s) {
    const int64_t groups = ((int64_t)a.rows.batch * a.heads + 7) / 8 * 8 * (OUT ? a.parts * (DV / 16) : (a.parts - 1) * ((DV + DK) / 16));
    constexpr int THREADS = OUT ? 512 : 256;
    constexpr int64_t LAUNCH = LAUNCH_GROUPS * 256 / THREADS;
    for (int64_t g = 0; g < groups; g += LAUNCH) {
        a.item0 = g;
        state_kernel<F32, DK, DV, OUT><<<dim3((unsigned)std::min(LAUNCH, groups - g)), dim3(THREADS), 0, s>>>(a, mats, parts);
    }
}

template <bool F32, int DK, int DV>
void launch_states(const DeltaArgs& a, const float* mats, float* parts, hipStream_t s) {
    if (a.parts > 1) launch_states<F32, DK, DV, false>(a, mats, parts, s);
    launch_states<F32, DK, DV, true>(a, mats, parts, s);
}

template <bool F32, int DK, int DV>
void launch_tokens(DeltaArgs a, hipStream_t s) {
    const int64_t groups = ((int64_t)a.rows.batch * a.heads * (DV / 32) + 3) / 4;
    for (int64_t g = 0; g < groups; g += LAUNCH_GROUPS) {
        a.item0 = g * 4;
        delta_token_kernel<F32, DK, DV><<<dim3((unsigned)std::min(LAUNCH_GROUPS, groups - g)), dim3(256), 0, s>>>(a);
    }
}

template <bool F32, int DK>
void launch_delta(const DeltaArgs& a, int dv, int64_t slots, float* mats, hipStream_t s) {
    if (slots) {
        launch_chunks<F32, DK>(a, slots, mats, s);
        float* const parts = mats + slots * a.heads * MATS;
        if (dv == 32) launch_states<F32, DK, 32>(a, mats, parts, s);
        else if (dv == 64) launch_states<F32, DK, 64>(a, mats, parts, s);
        else launch_states<F32, DK, 128>(a, mats, parts, s);
        return;
    }
    if (dv == 32) launch_tokens<F32, DK, 32>(a, s);
    else if (dv == 64) launch_tokens<F32, DK, 64>(a, s);
    else launch_tokens<F32, DK, 128>(a, s);
}

template <bool F32>
void launch_delta(const DeltaArgs& a, int dk, int dv, int64_t slots, float* mats, hipStream_t s) {
    if (dk == 32) launch_delta<F32, 32>(a, dv, slots, mats, s);
    else if (dk == 64) launch_delta<F32, 64>(a, dv, slots, mats, s);
    else launch_delta<F32, 128>(a, dv, slots, mats, s);
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
           s->k_stride >= qk && s->v_stride >= v && s->a_stride >= m->heads && s->b_stride >= m->heads &&
           std::max(s->q_stride, std::max(s->k_stride, s->v_stride)) <= (1 << 24);
}

}  // namespace

}  // namespace ssc

using namespace ssc;

extern "C" {

int sscater_delta_workspace(const sscater_delta_spec* spec, const sscater_delta_memory* memory,
                            const sscater_token_rows* rows, size_t* bytes) {
    if (!bytes || !delta_ok(spec, memory, rows)) return SSCATER_E_INVALID_ARG;
    *bytes = delta_bytes(delta_plan(memory, rows), memory);
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
    const DeltaPlan plan = delta_plan(memory, rows);
    const size_t need = delta_bytes(plan, memory);
    if (need > 0 && (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < need)) return SSCATER_E_INVALID_ARG;
    DeltaArgs x;
    // (no more than the streams can have: what lies behind them needs no workspace)
    x.rows.tokens = (int)std::min((int64_t)rows->tokens, (int64_t)rows->max_new * memory->batch); x.rows.max_new = rows->max_new; x.rows.batch = memory->batch;
    x.rows.start = rows->tokens ? rows->start : nullptr; x.rows.past = nullptr;
    x.from = initial ? initial : memory->state;
    x.state = memory->state;
    x.q = q; x.k = k; x.v = v; x.a = a; x.b = b; x.rate = rate; x.bias = bias; x.out = out;
    x.ldq = spec->q_stride; x.ldk = spec->k_stride; x.ldv = spec->v_stride; x.lda = spec->a_stride; x.ldb = spec->b_stride;
    x.heads = memory->heads; x.group = memory->heads / memory->qk_heads;
    x.unit = spec->unit; x.eps = spec->eps; x.scale = spec->scale; x.item0 = 0;
    x.parts = plan.parts; x.length = plan.length;
    float* const mats = (float*)workspace;
    if (size == 4) launch_delta<true>(x, memory->key_dim, memory->value_dim, plan.slots, mats, (hipStream_t)stream);
    else launch_delta<false>(x, memory->key_dim, memory->value_dim, plan.slots, mats, (hipStream_t)stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSCATER_OK : report_hip_error(e);
}

}  // extern "C"
