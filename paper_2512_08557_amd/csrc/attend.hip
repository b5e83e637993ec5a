// Attention of a call's new tokens over the token cache: a sliding window and
// the first tokens of the stream.
//
// Rows of a tile are (token, query head of one key head) pairs, token major, so
// the query heads that share a key head share the tile's keys.  The keys that
// some row of the tile sees form one range of "reach" positions u: the first
// min(sinks, LO) tokens of the stream, then LO, LO + 1, ...; u < sinks are
// exactly the sinks, and position u sits in slot u < sinks ? u : sinks +
// (base + u - sinks) mod ring.  Tiles of keys run over u, so sinks and window
// need no passes of their own.
//
// A wavefront owns 32 rows.  It forms the scores transposed, S^T = K Q^T, so a
// lane holds scores of one row (column lane % 32) and the running maximum and
// sum are one value per lane; O^T = V^T P^T then takes those scores as its
// second operand from the same registers: the keys of a matrix instruction may
// come in any order as long as V's come in the same one.  V is read from LDS
// with the transposing read (bf16).  exp is taken to base 2, sums in fp32;
// probabilities are rounded to bf16 for the product with bf16 values (as large
// as the output's own rounding), their sum is not.
//
// WM of the four wavefronts share keys and take different rows, the other
// 4 / WM groups take other tiles of keys and are joined at the end.  Where the
// rows leave compute units idle the keys are also split over workgroups, whose
// unnormalised sums are joined by a second launch.
#include "tokens.h"

#include <algorithm>

namespace ssc {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef short s4v __attribute__((ext_vector_type(4)));

struct AttendArgs {
    TokenRows rows;
    const void* q;
    const void* k;
    const void* v;
    void* out;
    float* part;           // [splits][tokens * q_heads][D] unnormalised sums, then [..][2] maximum and sum
    int q_heads, kv_heads, group;
    int sinks, capacity, window, causal;
    int qtiles, splits;
    float scale;           // times log2(e)
};

template <bool F32, int D, int WM>
struct AttendShape {
    static constexpr int S = F32 ? 4 : 2;
    static constexpr int RB = D * S;               // bytes of a cache row
    static constexpr int CPR = RB / 16;            // its 16-byte pieces
    static constexpr int BN = F32 ? 32 : 64;       // keys of a tile
    static constexpr int NT = BN / 32;
    static constexpr int TB = BN * RB;             // bytes of a tile
    static constexpr int WK = 4 / WM;              // groups over keys
    static constexpr int BM = 32 * WM;
    static constexpr int QN = RB / 32;             // 16-byte pieces of a lane's half of a query row
    static constexpr int ON = D / 2;               // output values of a lane
    static constexpr int LDS = WK * 2 * TB > 4 * ON * 256 || WK == 1 ? WK * 2 * TB : 4 * ON * 256;
    // Piece c of row r sits at piece c ^ swap: eight lanes that read one piece
    // of neighbouring rows (K), and the four rows of a transposed read (V, two
    // pieces each), fall on different banks.
    static __device__ __forceinline__ int swap_k(int r) { return CPR == 4 ? (r >> 1) & 3 : r & 7; }
    static __device__ __forceinline__ int swap_v(int r) { return F32 ? 0 : CPR == 4 ? r & 2 : (r & 3) * 2; }
};

// What a tile of rows reaches.
struct Reach {
    int total;             // positions u
    int base;              // ring offset of position u = sinks
    int n_sinks;           // sinks before LO
    int64_t lo;            // LO
};

__device__ __forceinline__ int slot_of(const AttendArgs& a, const Reach& r, int u) {
    if (u < a.sinks) return u;
    const int ring = a.capacity - a.sinks;
    int x = r.base + (u - a.sinks);
    if (x >= ring) x -= ring;
    return a.sinks + min(x, ring - 1);
}

template <bool F32, int D, int WM>
__global__ __launch_bounds__(256, 2) void attend_kernel(AttendArgs a) {
    using C = AttendShape<F32, D, WM>;
    __shared__ __attribute__((aligned(1024))) char lds[C::LDS];
    __shared__ float ml[4][32][2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = wave % WM, wk = wave / WM;
    const int h = lane >> 5, col = lane & 31;
    int id = blockIdx.x;
    const int split = id % a.splits;
    id /= a.splits;
    const int tile = id % a.qtiles;
    id /= a.qtiles;
    const int kvh = id % a.kv_heads, b = id / a.kv_heads;
    int first, n;
    rows_of(a.rows, b, first, n);
    const int nr = n * a.group;                    // rows of this key head
    if (tile * C::BM >= nr) return;
    const int64_t past = past_of(a.rows, b);
    const int i0 = tile * C::BM / a.group, i1 = (min((tile + 1) * C::BM, nr) - 1) / a.group;
    Reach reach;
    reach.lo = max((int64_t)0, (a.causal ? past + i0 : past) - a.window + 1);
    reach.n_sinks = (int)min((int64_t)a.sinks, reach.lo);
    reach.total = (int)min((int64_t)a.capacity,
                           reach.n_sinks + (a.causal ? past + i1 + 1 : past + n) - reach.lo);
    reach.base = (int)((max(reach.lo, (int64_t)a.sinks) - a.sinks) % (a.capacity - a.sinks));
    const int row = min(tile * C::BM + wm * 32 + col, nr - 1);
    const int tok = row / a.group;
    const int64_t qrow = ((int64_t)(first + tok) * a.q_heads + kvh * a.group + row % a.group);
    // the row sees u <= last, and of those u >= from or u < sinks
    const int last = (int)min((int64_t)reach.total - 1,
                              reach.n_sinks + (a.causal ? past + tok : past + n - 1) - reach.lo);
    const int from = (int)max((int64_t)0, reach.n_sinks + (a.causal ? past + tok : past) - a.window + 1 - reach.lo);

    uint4 qf[C::QN];
    {
        const char* p = (const char*)a.q + qrow * C::RB + h * 16;
#pragma unroll
        for (int s = 0; s < C::QN; ++s) qf[s] = *(const uint4*)(p + s * 32);
    }
    f16v o[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t) o[t] = f16v{};
    float m = -INFINITY, l = 0.f;

    const int tiles = (reach.total + C::BN - 1) / C::BN;
    const int per = (tiles + a.splits - 1) / a.splits;
    const int tb = min(tiles, split * per), te = min(tiles, tb + per);
    const int64_t head = ((int64_t)b * a.kv_heads + kvh) * a.capacity * C::RB;
    const char* kg = (const char*)a.k + head;
    const char* vg = (const char*)a.v + head;
    lds_char* kl = (lds_char*)lds + wk * 2 * C::TB;
    lds_char* vl = kl + C::TB;
    // rows of the wavefront that see least, for the choice of the masked form
    const int wl_first = __builtin_amdgcn_readfirstlane(last);
    const int wf_last = __builtin_amdgcn_readlane(from, 31);
    const int wl_last = __builtin_amdgcn_readlane(last, 31), wf_first = __builtin_amdgcn_readfirstlane(from);

    for (int t0 = tb; t0 < te; t0 += C::WK) {
        const int u0 = (t0 + wk) * C::BN;
        const bool live = t0 + wk < te;
        __syncthreads();
        if (live) {
            constexpr int RPC = 1024 / C::RB;      // rows of a copy
#pragma unroll
            for (int i = 0; i < C::TB / 1024 / WM; ++i) {
                const int c = i * WM + wm;
                const int r = c * RPC + lane / C::CPR, pc = lane % C::CPR;
                const int64_t at = (int64_t)slot_of(a, reach, min(u0 + r, reach.total - 1)) * C::RB;
                copy16(kg + at + (pc ^ C::swap_k(r)) * 16, kl + c * 1024);
                copy16(vg + at + (pc ^ C::swap_v(r)) * 16, vl + c * 1024);
            }
        }
        wait_vm<0>();
        __syncthreads();
        if (!live || u0 > wl_last || (u0 + C::BN <= wf_first && u0 >= a.sinks)) continue;
        f16v s[C::NT];
#pragma unroll
        for (int t = 0; t < C::NT; ++t) {
            s[t] = f16v{};
            const int r = 32 * t + col;
#pragma unroll
            for (int i = 0; i < C::QN; ++i) {
                const uint4 kf = lds16(kl + r * C::RB + ((2 * i + h) ^ C::swap_k(r)) * 16);
                if constexpr (F32) {
                    const uint32_t kv[4] = {kf.x, kf.y, kf.z, kf.w}, qv[4] = {qf[i].x, qf[i].y, qf[i].z, qf[i].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kv[e]), __uint_as_float(qv[e]), s[t],
                                                                    0, 0, 0);
                } else {
                    bf8v A, B;
                    __builtin_memcpy(&A, &kf, 16);
                    __builtin_memcpy(&B, &qf[i], 16);
                    s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(A, B, s[t], 0, 0, 0);
                }
            }
        }
        const bool masked = u0 + C::BN - 1 > wl_first || (u0 < wf_last && u0 + C::BN > a.sinks);
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < C::NT; ++t)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                float x = s[t][j] * a.scale;
                if (masked) {
                    const int u = u0 + 32 * t + 8 * (j >> 2) + 4 * h + (j & 3);
                    x = u <= last && (u >= from || u < a.sinks) ? x : -INFINITY;
                }
                s[t][j] = x;
                mx = fmaxf(mx, x);
            }
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float mn = fmaxf(m, mx), ms = mn == -INFINITY ? 0.f : mn;
        const float alpha = __builtin_amdgcn_exp2f(m - ms);
        m = mn;
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < C::NT; ++t)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                s[t][j] = __builtin_amdgcn_exp2f(s[t][j] - ms);
                sum += s[t][j];
            }
        l = l * alpha + sum;
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[t][j] *= alpha;
        bool plain = true;
        if (masked) {
            // A masked key's probability is zero, but its values may be
            // infinite or NaN: those tiles go key by key, past the masked ones.
            uint32_t big = 0;
            for (int i = lane; i < C::TB / 16; i += 64) {
                const uint4 v = lds16(vl + i * 16);
                for (uint32_t w : {v.x, v.y, v.z, v.w}) {
                    if constexpr (F32) big |= (w & 0x7F800000u) == 0x7F800000u;
                    else big |= ((w & 0x7F80u) == 0x7F80u) | ((w & 0x7F800000u) == 0x7F800000u);
                }
            }
            plain = __ballot(big != 0) == 0;
        }
        if (!plain) {
#pragma unroll 1
            for (int kk = 0; kk < C::BN; ++kk) {
                float p = 0.f;
#pragma unroll
                for (int e = 0; e < 16 * C::NT; ++e) {
                    const int key = 32 * (e >> 4) + 8 * ((e >> 2) & 3) + (e & 3);
                    if (key == (kk & ~4)) p = s[e >> 4][e & 15];
                }
                p = __shfl(p, col + 8 * (kk & 4));
                const int u = u0 + kk;
                const bool sees = u <= last && (u >= from || u < a.sinks);
#pragma unroll
                for (int e = 0; e < C::ON; ++e) {
                    const int d = 32 * (e >> 4) + 8 * ((e >> 2) & 3) + 4 * h + (e & 3);
                    const lds_char* at = vl + kk * C::RB + ((d * C::S / 16) ^ C::swap_v(kk)) * 16 + d * C::S % 16;
                    float v;
                    if constexpr (F32) v = *(const __attribute__((address_space(3))) float*)at;
                    else v = __uint_as_float((uint32_t)*(const __attribute__((address_space(3))) uint16_t*)at << 16);
                    if (sees) o[e >> 4][e & 15] = fmaf(p, v, o[e >> 4][e & 15]);
                }
            }
        } else if constexpr (F32) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int key = 8 * (j >> 2) + 4 * h + (j & 3);
#pragma unroll
                for (int t = 0; t < D / 32; ++t) {
                    const float v = *(const __attribute__((address_space(3))) float*)(vl + key * C::RB + (32 * t + col) * 4);
                    o[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[0][j], o[t], 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int ks = 0; ks < C::BN / 16; ++ks) {
                uint4 pf;
                const f16v& sv = s[ks / 2];
                const int j = 8 * (ks & 1);
                pf = make_uint4(bf16_pair(sv[j], sv[j + 1]), bf16_pair(sv[j + 2], sv[j + 3]),
                                bf16_pair(sv[j + 4], sv[j + 5]), bf16_pair(sv[j + 6], sv[j + 7]));
                bf8v B;
                __builtin_memcpy(&B, &pf, 16);
                const int i = lane & 15, key = 16 * ks + 4 * h + (i >> 2);
                // rows key and key + 8 have the same swap
                const lds_char* at = vl + key * C::RB + 8 * (i & 1);
#pragma unroll
                for (int t = 0; t < D / 32; ++t) {
                    const int c = (4 * t + 2 * ((lane >> 4) & 1) + ((i >> 1) & 1)) ^ C::swap_v(key);
                    typedef __attribute__((address_space(3))) s4v lds_s4v;
                    const s4v v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v*)(at + c * 16));
                    const s4v v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v*)(at + 8 * C::RB + c * 16));
                    bf8v A;
                    __builtin_memcpy(&A, &v0, 8);
                    __builtin_memcpy((char*)&A + 8, &v1, 8);
                    o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(A, B, o[t], 0, 0, 0);
                }
            }
        }
    }
    l += __shfl_xor(l, 32);

    int e0 = 0;
    constexpr int EN = C::ON / C::WK;              // output values that this lane writes
    if constexpr (C::WK > 1) {
        // the groups' sums through LDS; each group finishes a part of the values
        if (h == 0) {
            ml[wave][col][0] = m;
            ml[wave][col][1] = l;
        }
        __syncthreads();
        float* x = (float*)lds;
#pragma unroll
        for (int e = 0; e < C::ON; ++e) x[(wave * C::ON + e) * 64 + lane] = o[e >> 4][e & 15];
        __syncthreads();
        float big = -INFINITY;
#pragma unroll
        for (int g = 0; g < C::WK; ++g) big = fmaxf(big, ml[g * WM + wm][col][0]);
        const float ms = big == -INFINITY ? 0.f : big;
        float f[C::WK];
        l = 0.f;
#pragma unroll
        for (int g = 0; g < C::WK; ++g) {
            f[g] = __builtin_amdgcn_exp2f(ml[g * WM + wm][col][0] - ms);
            l += f[g] * ml[g * WM + wm][col][1];
        }
        m = big;
        e0 = wk * EN;
#pragma unroll
        for (int e = 0; e < EN; ++e) {
            float sum = 0.f;
#pragma unroll
            for (int g = 0; g < C::WK; ++g) sum = fmaf(f[g], x[((g * WM + wm) * C::ON + e0 + e) * 64 + lane], sum);
            o[e >> 4][e & 15] = sum;
        }
    }
    if (tile * C::BM + wm * 32 + col >= nr) return;
    const int64_t out_rows = (int64_t)a.rows.tokens * a.q_heads;
    const float r = a.splits > 1 ? 1.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < EN; e += 4) {
        const int g = e0 + e;
        const int d = 32 * (g >> 4) + 8 * ((g >> 2) & 3) + 4 * h;
        const f16v& ov = o[e >> 4];
        const int j = e & 15;
        const float v[4] = {ov[j] * r, ov[j + 1] * r, ov[j + 2] * r, ov[j + 3] * r};
        if (a.splits > 1) *(float4*)(a.part + (split * out_rows + qrow) * D + d) = make_float4(v[0], v[1], v[2], v[3]);
        else if constexpr (F32) *(float4*)((float*)a.out + qrow * D + d) = make_float4(v[0], v[1], v[2], v[3]);
        else *(uint2*)((uint16_t*)a.out + qrow * D + d) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
    }
    if (a.splits > 1 && h == 0 && wk == 0)
        *(float2*)(a.part + a.splits * out_rows * D + (split * out_rows + qrow) * 2) = make_float2(m, l);
}

// The splits' sums of one row, joined: D / 4 lanes a row.
template <bool F32, int D>
__global__ __launch_bounds__(256) void join_kernel(const float* part, void* out, int64_t rows, int splits) {
    const int64_t row = (int64_t)blockIdx.x * (1024 / D) + threadIdx.x / (D / 4);
    if (row >= rows) return;
    const int d = threadIdx.x % (D / 4) * 4;
    const float* ml = part + splits * rows * D + row * 2;
    float big = -INFINITY;
    for (int s = 0; s < splits; ++s) big = fmaxf(big, ml[s * rows * 2]);
    const float ms = big == -INFINITY ? 0.f : big;
    float l = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < splits; ++s) {
        const float f = __builtin_amdgcn_exp2f(ml[s * rows * 2] - ms);
        const float4 p = *(const float4*)(part + (s * rows + row) * D + d);
        l = fmaf(f, ml[s * rows * 2 + 1], l);
        v[0] = fmaf(f, p.x, v[0]);
        v[1] = fmaf(f, p.y, v[1]);
        v[2] = fmaf(f, p.z, v[2]);
        v[3] = fmaf(f, p.w, v[3]);
    }
    const float r = 1.f / l;
    if constexpr (F32) *(float4*)((float*)out + row * D + d) = make_float4(v[0] * r, v[1] * r, v[2] * r, v[3] * r);
    else *(uint2*)((uint16_t*)out + row * D + d) = make_uint2(bf16_pair(v[0] * r, v[1] * r), bf16_pair(v[2] * r, v[3] * r));
}

namespace {

// How a call is cut up, from what the host knows.
struct AttendCut {
    int wm, qtiles, splits;
    int64_t grid;
};

bool attend_cut(const sscater_attend_spec* s, const sscater_token_cache* c, const sscater_token_rows* r, AttendCut* cut) {
    if (!s || !token_cache_ok(c) || !token_rows_ok(c, r)) return false;
    if (s->q_heads < 1 || s->q_heads > (1 << 16) || s->q_heads % c->kv_heads || s->window < 1 || s->causal < 0 ||
        s->causal > 1 || !(s->scale == s->scale))
        return false;
    const int64_t reach = std::min((int64_t)s->window + r->max_new - 1, r->max_past + r->max_new);
    if (r->tokens > 0 && c->capacity - c->sinks < reach) return false;
    const int64_t rows = (int64_t)r->max_new * (s->q_heads / c->kv_heads);
    if (rows > (1 << 30) || (int64_t)r->tokens * s->q_heads > (int64_t(1) << 40)) return false;
    cut->wm = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
    cut->qtiles = (int)((rows + 32 * cut->wm - 1) / (32 * cut->wm));
    const int64_t base = (int64_t)cut->qtiles * c->kv_heads * c->batch;
    const int64_t keys = reach + c->sinks;
    const int bn = (c->dtype == SSCATER_F32 ? 32 : 64) * (4 / cut->wm);
    cut->splits = 1;
    if (base > 0 && base < 256)
        cut->splits = (int)std::max((int64_t)1, std::min((512 + base - 1) / base, (keys + 2 * bn - 1) / (2 * bn)));
    cut->grid = base * cut->splits;
    return cut->grid <= 0x7FFFFFFF;
}

size_t attend_bytes(const AttendCut& cut, const sscater_attend_spec* s, const sscater_token_cache* c,
                    const sscater_token_rows* r) {
    return cut.splits > 1 ? (size_t)cut.splits * r->tokens * s->q_heads * (c->head_dim + 2) * 4 : 0;
}

template <bool F32, int D>
void launch_attend(const AttendArgs& a, const AttendCut& cut, hipStream_t s) {
    const dim3 grid((unsigned)cut.grid), block(256);
    if (cut.wm == 1) attend_kernel<F32, D, 1><<<grid, block, 0, s>>>(a);
    else if (cut.wm == 2) attend_kernel<F32, D, 2><<<grid, block, 0, s>>>(a);
    else attend_kernel<F32, D, 4><<<grid, block, 0, s>>>(a);
    if (cut.splits > 1) {
        const int64_t rows = (int64_t)a.rows.tokens * a.q_heads;
        join_kernel<F32, D><<<dim3((unsigned)((rows + 1024 / D - 1) / (1024 / D))), block, 0, s>>>(a.part, a.out, rows,
                                                                                                  cut.splits);
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
    a.scale = spec->scale * 1.4426950408889634f;
    if (cache->dtype == SSCATER_F32) launch_attend<true>(a, cut, cache->head_dim, (hipStream_t)stream);
    else launch_attend<false>(a, cut, cache->head_dim, (hipStream_t)stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSCATER_OK : report_hip_error(e);
}

}  // extern "C"
