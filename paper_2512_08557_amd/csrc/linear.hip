// Linear layers over rows of cells: y = act(x W^T + b) + r.
//
// A workgroup of four wavefronts owns a tile of 128 rows and 128 output
// channels, a wavefront 64 x 64 of it as 2 x 2 blocks of 32 x 32.  K runs in
// steps through two LDS stages.  W is the first matrix operand and x the
// second, so a lane holds four consecutive output channels of one row.
//
// fp32: a step's values are split in registers into three bf16 planes of 8
// bits each by cutting off (h + m + l is the value exactly), and six of the
// nine products are formed; the others are at most 2^-23 of the whole.
#include <hip/hip_runtime.h>

#include "../../include/sscater.h"
#include "device_common.h"

namespace ssc {

typedef float f16v __attribute__((ext_vector_type(16)));

struct LinearArgs {
    const void* x;
    const void* w;
    const void* bias;
    const void* res;
    void* y;
    int64_t M, ldx, ldw, ldr, ldy;
    int K, N, act;
    int tn;               // tiles across the output channels
    int tiles, per_xcd;   // all tiles, and those of an XCD (workgroup b runs on XCD b % 8)
    int rvec, yvec;       // residual and output rows may be accessed 16 bytes at a time
};

// Up to this many rows take linear_rows_kernel.
constexpr int ROWS_KERNEL = 64;

// What a copy reads where its tile has nothing.
__device__ __attribute__((aligned(16))) uint32_t linear_zero[4];

// z (1 + erf(z / sqrt 2)) / 2, with erfc(t) = exp(-t^2) p(1 / (1 + 0.3275911 t))
// for t >= 0 (Abramowitz and Stegun 7.1.26, |error| <= 1.5e-7).
__device__ __forceinline__ float gelu(float z) {
    const float t = fabsf(z) * 0.70710678f;
    const float u = __builtin_amdgcn_rcpf(fmaf(0.3275911f, t, 1.f));
    float p = fmaf(1.061405429f, u, -1.453152027f);
    p = fmaf(p, u, 1.421413741f);
    p = fmaf(p, u, -0.284496736f);
    p = fmaf(p, u, 0.254829592f) * u;
    const float half = 0.5f * z * (p * __builtin_amdgcn_exp2f(-1.44269504f * t * t));
    return z >= 0.f ? z - half : half;
}

__device__ __forceinline__ float activate(float z, int act) {
    if (act == SSCATER_ACT_RELU) return z < 0.f ? 0.f : z;
    if (act == SSCATER_ACT_GELU) return fabsf(z) > 1e30f ? fmaxf(z, 0.f) : gelu(z);
    if (act == SSCATER_ACT_SILU) return z / (1.f + __expf(-z));
    return z;
}

template <bool F32>
__device__ __forceinline__ float load_value(const void* p, int64_t i) {
    if constexpr (F32) return ((const float*)p)[i];
    return __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16);
}

// The three planes of two values by cutting off: x in the low halves.
__device__ __forceinline__ void cut_pair(uint32_t x, uint32_t y, uint32_t& h, uint32_t& m, uint32_t& l) {
    const float rx = __uint_as_float(x) - __uint_as_float(x & 0xFFFF0000u);
    const float ry = __uint_as_float(y) - __uint_as_float(y & 0xFFFF0000u);
    h = __builtin_amdgcn_perm(y, x, 0x07060302u);
    const uint32_t ux = __float_as_uint(rx), uy = __float_as_uint(ry);
    m = __builtin_amdgcn_perm(uy, ux, 0x07060302u);
    const float sx = rx - __uint_as_float(ux & 0xFFFF0000u), sy = ry - __uint_as_float(uy & 0xFFFF0000u);
    l = __builtin_amdgcn_perm(__float_as_uint(sy), __float_as_uint(sx), 0x07060302u);
}

__device__ __forceinline__ f16v mfma32(uint4 a, uint4 b, f16v c) {
    bf8v A, B;
    __builtin_memcpy(&A, &a, 16);
    __builtin_memcpy(&B, &b, 16);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(A, B, c, 0, 0, 0);
}

// 16-byte piece `piece` of tile row `row` in LDS: rows of RB bytes, the pieces
// of neighbouring rows moved so that lanes which read one piece of eight rows
// fall on different banks.
template <int RB>
__device__ __forceinline__ int place(int row, int piece) {
    if constexpr (RB == 64) return row * 64 + ((piece ^ (row >> 1)) & 3) * 16;
    return row * 128 + ((piece ^ row) & 7) * 16;
}

// One K step of an operand tile as 16-byte pieces in registers, for rows that
// are split (fp32) or may not be read 16 bytes at a time (not VEC): piece i of
// the thread is row (tid + 256 i) / P, piece (tid + 256 i) % P of it.
template <bool F32, bool VEC, int ROWS, int P>
struct Staged {
    static constexpr int E = F32 ? 4 : 8, N = ROWS * P / 256;
    uint4 v[N];
    __device__ __forceinline__ void load(const void* base, int64_t ld, int64_t row0, int64_t rows, int k0, int K) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = threadIdx.x + 256 * i;
            const int64_t row = min(row0 + at / P, rows - 1);
            const int k = k0 + at % P * E;
            if constexpr (VEC) {
                v[i] = make_uint4(0, 0, 0, 0);
                if (k < K) v[i] = *(const uint4*)((const char*)base + (row * ld + k) * (F32 ? 4 : 2));
            } else {
                uint32_t b[4] = {0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if (k + e >= K) continue;
                    if constexpr (F32) b[e] = ((const uint32_t*)base)[row * ld + k + e];
                    else b[e / 2] |= (uint32_t)((const uint16_t*)base)[row * ld + k + e] << (16 * (e & 1));
                }
                v[i] = make_uint4(b[0], b[1], b[2], b[3]);
            }
        }
    }
    // bf16: as it is; fp32: three planes of ROWS rows of 64 bytes
    __device__ __forceinline__ void store(lds_char* lds) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = threadIdx.x + 256 * i, row = at / P, c = at % P;
            if constexpr (F32) {
                uint32_t h[2], m[2], l[2];
                cut_pair(v[i].x, v[i].y, h[0], m[0], l[0]);
                cut_pair(v[i].z, v[i].w, h[1], m[1], l[1]);
                lds_char* to = lds + place<64>(row, c >> 1) + (c & 1) * 8;
                store8(to, h);
                store8(to + ROWS * 64, m);
                store8(to + 2 * ROWS * 64, l);
            } else {
                typedef uint32_t u4v __attribute__((ext_vector_type(4)));
                *(__attribute__((address_space(3))) u4v*)(lds + place<16 * P>(row, c)) =
                    u4v{v[i].x, v[i].y, v[i].z, v[i].w};
            }
        }
    }
    static __device__ __forceinline__ void store8(lds_char* to, const uint32_t (&w)[2]) {
        typedef uint32_t u2v __attribute__((ext_vector_type(2)));
        *(__attribute__((address_space(3))) u2v*)to = u2v{w[0], w[1]};
    }
};

// The same straight into LDS (bf16 rows on 16-byte boundaries): a copy is 1 KB,
// the four wavefronts take them in turn.
template <int ROWS, int P>
__device__ __forceinline__ void copy_tile(lds_char* lds, const void* base, int64_t ld, int64_t row0, int64_t rows,
                                          int k0, int K) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < ROWS * P / 256; ++i) {
        const int c = i * 4 + wave;
        const int row = c * (64 / P) + lane / P;
        const int piece = (lane % P) ^ (P == 4 ? (row >> 1) & 3 : row & 7);
        const int k = k0 + piece * 8;
        const char* src = (const char*)base + (min(row0 + row, rows - 1) * ld + k) * 2;
        copy16(k < K ? src : (const char*)linear_zero, lds + c * 1024);
    }
}

// E values of a row: bias, activation, residual, rounding.
template <bool F32>
__device__ __forceinline__ void finish(const LinearArgs& a, float (&z)[8], const float (&bias)[8], int64_t m, int n) {
    constexpr int E = 8;
#pragma unroll
    for (int e = 0; e < E; ++e) z[e] += bias[e];
    if (a.act == SSCATER_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < E; ++e) z[e] = activate(z[e], SSCATER_ACT_RELU);
    } else if (a.act == SSCATER_ACT_GELU) {
#pragma unroll
        for (int e = 0; e < E; ++e) z[e] = activate(z[e], SSCATER_ACT_GELU);
    } else if (a.act == SSCATER_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < E; ++e) z[e] = activate(z[e], SSCATER_ACT_SILU);
    }
    const bool whole = n + E <= a.N;
    if (a.res) {
        if (whole && a.rvec) {
            if constexpr (F32) {
                const float4* r = (const float4*)((const float*)a.res + m * a.ldr + n);
                const float4 r0 = r[0], r1 = r[1];
                z[0] += r0.x; z[1] += r0.y; z[2] += r0.z; z[3] += r0.w;
                z[4] += r1.x; z[5] += r1.y; z[6] += r1.z; z[7] += r1.w;
            } else {
                const uint4 r = *(const uint4*)((const uint16_t*)a.res + m * a.ldr + n);
                const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    z[2 * e] += __uint_as_float(w[e] << 16);
                    z[2 * e + 1] += __uint_as_float(w[e] & 0xFFFF0000u);
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (n + e < a.N) z[e] += load_value<F32>(a.res, m * a.ldr + n + e);
        }
    }
    if (whole && a.yvec) {
        if constexpr (F32) {
            float4* y = (float4*)((float*)a.y + m * a.ldy + n);
            y[0] = make_float4(z[0], z[1], z[2], z[3]);
            y[1] = make_float4(z[4], z[5], z[6], z[7]);
        } else {
            *(uint4*)((uint16_t*)a.y + m * a.ldy + n) = make_uint4(bf16_pair(z[0], z[1]), bf16_pair(z[2], z[3]),
                                                                   bf16_pair(z[4], z[5]), bf16_pair(z[6], z[7]));
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (n + e < a.N) {
                if constexpr (F32) ((float*)a.y)[m * a.ldy + n + e] = z[e];
                else ((uint16_t*)a.y)[m * a.ldy + n + e] = (uint16_t)bf16_pair(z[e], z[e]);
            }
    }
}

// A wavefront owns TM x TN blocks of 32 rows x 32 output channels, the
// workgroup WM x WN (= 4) wavefronts.
template <bool F32, bool VEC, int WM, int WN, int TM, int TN>
struct LinearShape {
    static constexpr int BM = 32 * WM * TM, BN = 32 * WN * TN;
    static constexpr bool COPY = VEC && !F32;          // straight into LDS
    static constexpr int P = F32 ? 8 : 8;              // 16-byte pieces of a row's K step
    static constexpr int BK = P * (F32 ? 4 : 8);       // 32 or 64 channels
    static constexpr int SX = F32 ? BM * 64 * 3 : BM * 16 * P;
    static constexpr int SW = F32 ? BN * 64 * 3 : BN * 16 * P;
    static constexpr int NST = COPY ? 2 : 1;           // stages in LDS
    static constexpr int PITCH = 32 * TN + 4;          // floats of a row on the way out
    static constexpr int OUT = 4 * 32 * PITCH * 4;
    static constexpr int LDS = NST * (SX + SW) > OUT ? NST * (SX + SW) : OUT;
};

template <bool F32, bool VEC, int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(256, 2) void linear_kernel(LinearArgs a) {
    using C = LinearShape<F32, VEC, WM, WN, TM, TN>;
    __shared__ __attribute__((aligned(1024))) char lds_[C::LDS];
    lds_char* lds = (lds_char*)lds_;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int id = (int)(blockIdx.x & 7) * a.per_xcd + (int)(blockIdx.x >> 3);
    if (id >= a.tiles) return;
    const int64_t m0 = (int64_t)(id / a.tn) * C::BM;
    const int n0 = (id % a.tn) * C::BN;
    const int wm = wave % WM * (32 * TM), wn = wave / WM * (32 * TN);
    const int r = lane & 31, h = lane >> 5;
    f16v acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = f16v{};

    auto multiply = [&](const lds_char* X, const lds_char* W) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < C::BK / 16; ++s) {
            if constexpr (F32) {
                uint4 x[TM][3], w[TN][3];
#pragma unroll
                for (int p = 0; p < 3; ++p) {
#pragma unroll
                    for (int j = 0; j < TM; ++j)
                        x[j][p] = lds16(X + p * C::BM * 64 + place<64>(wm + 32 * j + r, 2 * s + h));
#pragma unroll
                    for (int i = 0; i < TN; ++i)
                        w[i][p] = lds16(W + p * C::BN * 64 + place<64>(wn + 32 * i + r, 2 * s + h));
                }
#pragma unroll
                for (int t = 0; t < 6; ++t) {
                    constexpr int PW[6] = {2, 0, 1, 1, 0, 0}, PX[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
                    for (int i = 0; i < TN; ++i)
#pragma unroll
                        for (int j = 0; j < TM; ++j) acc[i][j] = mfma32(w[i][PW[t]], x[j][PX[t]], acc[i][j]);
                }
            } else {
                uint4 x[TM], w[TN];
#pragma unroll
                for (int j = 0; j < TM; ++j) x[j] = lds16(X + place<16 * C::P>(wm + 32 * j + r, 2 * s + h));
#pragma unroll
                for (int i = 0; i < TN; ++i) w[i] = lds16(W + place<16 * C::P>(wn + 32 * i + r, 2 * s + h));
#pragma unroll
                for (int i = 0; i < TN; ++i)
#pragma unroll
                    for (int j = 0; j < TM; ++j) acc[i][j] = mfma32(w[i], x[j], acc[i][j]);
            }
        }
    };

    if constexpr (C::COPY) {
        constexpr int CP = (C::BM + C::BN) * C::P / 256;     // copies of a wavefront per stage
        auto issue = [&](int step) __attribute__((always_inline)) {
            lds_char* to = lds + (step & 1) * (C::SX + C::SW);
            copy_tile<C::BM, C::P>(to, a.x, a.ldx, m0, a.M, step * C::BK, a.K);
            copy_tile<C::BN, C::P>(to + C::SX, a.w, a.ldw, n0, a.N, step * C::BK, a.K);
        };
        const int steps = (a.K + C::BK - 1) / C::BK;
        issue(0);
        for (int k = 0; k < steps; ++k) {
            if (k + 1 < steps) {
                issue(k + 1);
                wait_vm<CP>();
            } else {
                wait_vm<0>();
            }
            lds_barrier();
            const lds_char* X = lds + (k & 1) * (C::SX + C::SW);
            multiply(X, X + C::SX);
            lds_barrier();
        }
    } else {
        Staged<F32, VEC, C::BM, C::P> x;
        Staged<F32, VEC, C::BN, C::P> w;
        x.load(a.x, a.ldx, m0, a.M, 0, a.K);
        w.load(a.w, a.ldw, n0, a.N, 0, a.K);
        for (int k0 = 0; k0 < a.K; k0 += C::BK) {
            x.store(lds);
            w.store(lds + C::SX);
            __syncthreads();
            if (k0 + C::BK < a.K) {
                x.load(a.x, a.ldx, m0, a.M, k0 + C::BK, a.K);
                w.load(a.w, a.ldw, n0, a.N, k0 + C::BK, a.K);
            }
            multiply(lds, lds + C::SX);
            __syncthreads();
        }
    }

    // On the way out the wavefront's sums pass through its own part of LDS, 32
    // rows at a time, so that a row's channels are stored together.
    constexpr int G = 4 * TN;                          // lanes of a row
    float* t = (float*)lds_ + wave * 32 * C::PITCH;
    const int n = n0 + wn + lane % G * 8;
    float bias[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = a.bias && n + e < a.N ? load_value<F32>(a.bias, n + e) : 0.f;
#pragma unroll
    for (int j = 0; j < TM; ++j) {
        const int64_t mb = m0 + wm + 32 * j;
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float z[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    z[e] = acc[i][j][4 * g + e];
                    const int nn = n0 + wn + 32 * i + 8 * g + 4 * h + e;
                    if (F32 && z[e] != z[e] && nn < a.N && mb + r < a.M) {
                        // an infinity leaves a NaN in its lower planes: such a sum is formed again from the values
                        z[e] = 0.f;
                        for (int k = 0; k < a.K; ++k)
                            z[e] = fmaf(load_value<F32>(a.x, (mb + r) * a.ldx + k), load_value<F32>(a.w, nn * a.ldw + k),
                                        z[e]);
                    }
                }
                *(float4*)(t + r * C::PITCH + 32 * i + 8 * g + 4 * h) = make_float4(z[0], z[1], z[2], z[3]);
            }
#pragma unroll
        for (int p = 0; p < 32 / (64 / G); ++p) {
            const int row = p * (64 / G) + lane / G;
            const float4 z0 = *(const float4*)(t + row * C::PITCH + lane % G * 8);
            const float4 z1 = *(const float4*)(t + row * C::PITCH + lane % G * 8 + 4);
            float z[8] = {z0.x, z0.y, z0.z, z0.w, z1.x, z1.y, z1.z, z1.w};
            if (mb + row < a.M && n < a.N) finish<F32>(a, z, bias, mb + row, n);
        }
    }
}

// Few rows: a workgroup owns 16 rows x 16 output channels and its wavefronts
// share K, each with its operands straight from memory, so that a call is one
// round trip and a sum through LDS.  fp32 takes the fp32 matrix instructions.
template <bool F32, bool VEC>
__global__ __launch_bounds__(256) void linear_rows_kernel(LinearArgs a) {
    constexpr int E = F32 ? 4 : 8, BK = 4 * E;         // channels of a lane, and of a wavefront's piece
    __shared__ float sums[4][4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n0 = (int)(blockIdx.x % a.tn) * 16;
    const int64_t m0 = (int64_t)(blockIdx.x / a.tn) * 16;
    const int64_t n = min(n0 + (lane & 15), a.N - 1), m = min(m0 + (lane & 15), a.M - 1);
    const int64_t xo = m * a.ldx, wo = n * a.ldw;
    f4v acc = {0.f, 0.f, 0.f, 0.f};
    auto load = [&](const void* p, int64_t o, int k) __attribute__((always_inline)) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if constexpr (VEC) {
            if (k < a.K) v = *(const uint4*)((const char*)p + (o + k) * (F32 ? 4 : 2));
        } else {
            uint32_t b[4] = {0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (k + e >= a.K) continue;
                if constexpr (F32) b[e] = ((const uint32_t*)p)[o + k + e];
                else b[e / 2] |= (uint32_t)((const uint16_t*)p)[o + k + e] << (16 * (e & 1));
            }
            v = make_uint4(b[0], b[1], b[2], b[3]);
        }
        return v;
    };
    constexpr int U = VEC ? 4 : 2;                     // pieces in flight
    for (int k0 = wave * BK; k0 < a.K; k0 += 4 * BK * U) {
        uint4 x[U], w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = k0 + u * 4 * BK + (lane >> 4) * E;
            w[u] = load(a.w, wo, k);
            x[u] = load(a.x, xo, k);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if constexpr (F32) {
                const uint32_t wv[4] = {w[u].x, w[u].y, w[u].z, w[u].w}, xv[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(wv[e]), __uint_as_float(xv[e]), acc, 0, 0, 0);
            } else {
                acc = mfma_bf16(w[u], x[u], acc);
            }
        }
    }
    // lane l, register j: channel 4 (l / 16) + j of row l % 16
#pragma unroll
    for (int j = 0; j < 4; ++j) sums[wave][j][lane] = acc[j];
    __syncthreads();
    const int c = threadIdx.x & 15, row = threadIdx.x >> 4;
    const int at = (c >> 2) * 16 + row;
    if (n0 + c >= a.N || m0 + row >= a.M) return;
    float z = (sums[0][c & 3][at] + sums[1][c & 3][at]) + (sums[2][c & 3][at] + sums[3][c & 3][at]);
    if (a.bias) z += load_value<F32>(a.bias, n0 + c);
    z = activate(z, a.act);
    if (a.res) z += load_value<F32>(a.res, (m0 + row) * a.ldr + n0 + c);
    if constexpr (F32) ((float*)a.y)[(m0 + row) * a.ldy + n0 + c] = z;
    else ((uint16_t*)a.y)[(m0 + row) * a.ldy + n0 + c] = (uint16_t)bf16_pair(z, z);
}

namespace {

template <bool F32, bool VEC, int WM, int WN, int TM, int TN>
bool launch_tiles(LinearArgs& a, hipStream_t s) {
    using C = LinearShape<F32, VEC, WM, WN, TM, TN>;
    a.tn = (a.N + C::BN - 1) / C::BN;
    const int64_t tiles = (a.M + C::BM - 1) / C::BM * a.tn;
    if (tiles > 0x7FFFFFF0) return false;
    a.tiles = (int)tiles;
    a.per_xcd = (int)((tiles + 7) / 8);
    linear_kernel<F32, VEC, WM, WN, TM, TN><<<dim3((unsigned)a.per_xcd * 8), dim3(256), 0, s>>>(a);
    return true;
}

template <bool F32, bool VEC>
bool launch_linear(LinearArgs& a, hipStream_t s) {
    if (a.M <= ROWS_KERNEL) {
        a.tn = (a.N + 15) / 16;
        const int64_t grid = (a.M + 15) / 16 * a.tn;
        linear_rows_kernel<F32, VEC><<<dim3((unsigned)grid), dim3(256), 0, s>>>(a);
        return true;
    }
    const int64_t big = ((a.M + 127) / 128) * ((a.N + 127) / 128);
    if (a.N <= 64 && a.M >= 256 * 64) return launch_tiles<F32, VEC, 4, 1, 1, 2>(a, s);
    if (big >= 256 && a.N > 64) return launch_tiles<F32, VEC, 2, 2, 2, 2>(a, s);
    return launch_tiles<F32, VEC, 2, 2, 1, 1>(a, s);
}

}  // namespace

}  // namespace ssc

using namespace ssc;

extern "C" int sscater_linear(const sscater_linear_spec* spec, const void* x, const void* weight, const void* bias,
                              const void* residual, void* y, void* stream) {
    if (!spec || spec->rows < 0 || spec->cin < 1 || spec->cout < 1) return SSCATER_E_INVALID_ARG;
    if (spec->dtype != SSCATER_F32 && spec->dtype != SSCATER_BF16) return SSCATER_E_INVALID_ARG;
    if (spec->activation < SSCATER_ACT_NONE || spec->activation > SSCATER_ACT_SILU) return SSCATER_E_INVALID_ARG;
    if (spec->rows > (int64_t(1) << 36) || spec->cin > (1 << 30) || spec->cout > (1 << 30)) return SSCATER_E_INVALID_ARG;
    if (spec->x_stride < spec->cin || spec->w_stride < spec->cin || spec->y_stride < spec->cout ||
        (residual && spec->residual_stride < spec->cout))
        return SSCATER_E_INVALID_ARG;
    if (spec->rows == 0) return SSCATER_OK;
    const int size = spec->dtype == SSCATER_F32 ? 4 : 2;
    for (const void* p : {x, weight, (const void*)y})
        if (!p || (uintptr_t)p % size) return SSCATER_E_INVALID_ARG;
    for (const void* p : {bias, residual})
        if ((uintptr_t)p % size) return SSCATER_E_INVALID_ARG;
    LinearArgs a;
    a.x = x; a.w = weight; a.bias = bias; a.res = residual; a.y = y;
    a.M = spec->rows; a.K = spec->cin; a.N = spec->cout; a.act = spec->activation;
    a.ldx = spec->x_stride; a.ldw = spec->w_stride; a.ldr = spec->residual_stride; a.ldy = spec->y_stride;
    const int per = 16 / size;
    const bool vec = (uintptr_t)x % 16 == 0 && (uintptr_t)weight % 16 == 0 && a.K % per == 0 && a.ldx % per == 0 &&
                     a.ldw % per == 0;
    a.yvec = (uintptr_t)y % 16 == 0 && a.ldy % per == 0;
    a.rvec = (uintptr_t)residual % 16 == 0 && a.ldr % per == 0;
    const hipStream_t s = (hipStream_t)stream;
    const bool fits = size == 4 ? vec ? launch_linear<true, true>(a, s) : launch_linear<true, false>(a, s)
                                : vec ? launch_linear<false, true>(a, s) : launch_linear<false, false>(a, s);
    if (!fits) return SSCATER_E_INVALID_ARG;
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSCATER_OK : report_hip_error(e);
}
