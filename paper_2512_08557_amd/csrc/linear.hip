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
};

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

constexpr int LT = 128;                       // tile edge

// Four 16-byte pieces of an operand tile's K step (rows of 128 bytes) into
// registers: piece i of the thread is row (tid + 256 i) / 8, bytes 16 * (tid % 8).
template <bool F32, bool VEC>
__device__ __forceinline__ void load_pieces(uint4 (&v)[4], const void* base, int64_t ld, int64_t row0, int64_t rows,
                                            int k0, int K) {
    constexpr int E = F32 ? 4 : 8;
    const int c = threadIdx.x & 7;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        int64_t row = row0 + (threadIdx.x >> 3) + 32 * i;
        row = row < rows ? row : rows - 1;
        const int k = k0 + c * E;
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

// bf16 rows of 128 bytes (64 channels): piece c of row r at r * 128 + ((c ^ r) & 7) * 16.
__device__ __forceinline__ int place128(int row, int piece) { return row * 128 + ((piece ^ row) & 7) * 16; }
// planes' rows of 64 bytes (32 channels): piece c of row r at r * 64 + ((c ^ (r >> 1)) & 3) * 16.
__device__ __forceinline__ int place64(int row, int piece) { return row * 64 + ((piece ^ (row >> 1)) & 3) * 16; }

template <bool F32>
__device__ __forceinline__ void store_pieces(char* lds, const uint4 (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = (threadIdx.x >> 3) + 32 * i, c = threadIdx.x & 7;
        if constexpr (F32) {
            uint32_t h[2], m[2], l[2];
            cut_pair(v[i].x, v[i].y, h[0], m[0], l[0]);
            cut_pair(v[i].z, v[i].w, h[1], m[1], l[1]);
            const int at = place64(row, c >> 1) + (c & 1) * 8;
            *(uint2*)(lds + at) = make_uint2(h[0], h[1]);
            *(uint2*)(lds + LT * 64 + at) = make_uint2(m[0], m[1]);
            *(uint2*)(lds + 2 * LT * 64 + at) = make_uint2(l[0], l[1]);
        } else {
            *(uint4*)(lds + place128(row, c)) = v[i];
        }
    }
}

template <bool F32, bool VEC>
__global__ __launch_bounds__(256) void linear_kernel(LinearArgs a) {
    constexpr int BK = F32 ? 32 : 64;
    constexpr int OPB = F32 ? LT * 64 * 3 : LT * 128;      // bytes of an operand's stage
    __shared__ __attribute__((aligned(1024))) char lds[2 * OPB];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t m0 = (int64_t)(blockIdx.x / a.tn) * LT;
    const int n0 = (int)(blockIdx.x % a.tn) * LT;
    const int wm = (wave & 1) * 64, wn = (wave >> 1) * 64;
    f16v acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = f16v{};
    uint4 vx[4], vw[4];
    load_pieces<F32, VEC>(vx, a.x, a.ldx, m0, a.M, 0, a.K);
    load_pieces<F32, VEC>(vw, a.w, a.ldw, n0, a.N, 0, a.K);
    for (int k0 = 0; k0 < a.K; k0 += BK) {
        __syncthreads();
        store_pieces<F32>(lds, vx);
        store_pieces<F32>(lds + OPB, vw);
        __syncthreads();
        if (k0 + BK < a.K) {
            load_pieces<F32, VEC>(vx, a.x, a.ldx, m0, a.M, k0 + BK, a.K);
            load_pieces<F32, VEC>(vw, a.w, a.ldw, n0, a.N, k0 + BK, a.K);
        }
        const int r = lane & 31, h = lane >> 5;
#pragma unroll
        for (int s = 0; s < BK / 16; ++s) {
            if constexpr (F32) {
                uint4 X[2][3], W[2][3];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int p = 0; p < 3; ++p) {
                        X[i][p] = *(const uint4*)(lds + p * LT * 64 + place64(wm + 32 * i + r, 2 * s + h));
                        W[i][p] = *(const uint4*)(lds + OPB + p * LT * 64 + place64(wn + 32 * i + r, 2 * s + h));
                    }
#pragma unroll
                for (int t = 0; t < 6; ++t) {
                    constexpr int PW[6] = {2, 0, 1, 1, 0, 0}, PX[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int j = 0; j < 2; ++j) acc[i][j] = mfma32(W[i][PW[t]], X[j][PX[t]], acc[i][j]);
                }
            } else {
                uint4 X[2], W[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    X[i] = *(const uint4*)(lds + place128(wm + 32 * i + r, 2 * s + h));
                    W[i] = *(const uint4*)(lds + OPB + place128(wn + 32 * i + r, 2 * s + h));
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = mfma32(W[i], X[j], acc[i][j]);
            }
        }
    }
    const int r = lane & 31, h = lane >> 5;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t m = m0 + wm + 32 * j + r;
        if (m >= a.M) continue;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int n = n0 + wn + 32 * i + 8 * (e >> 2) + 4 * h + (e & 3);
                if (n >= a.N) continue;
                float z = acc[i][j][e];
                if (F32 && z != z) {
                    // an infinity leaves a NaN in its lower planes: such a sum is formed again from the values
                    z = 0.f;
                    for (int k = 0; k < a.K; ++k)
                        z = fmaf(load_value<F32>(a.x, m * a.ldx + k), load_value<F32>(a.w, n * a.ldw + k), z);
                }
                if (a.bias) z += load_value<F32>(a.bias, n);
                z = activate(z, a.act);
                if (a.res) z += load_value<F32>(a.res, m * a.ldr + n);
                if constexpr (F32) ((float*)a.y)[m * a.ldy + n] = z;
                else ((uint16_t*)a.y)[m * a.ldy + n] = (uint16_t)bf16_pair(z, z);
            }
    }
}

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
    a.tn = (a.N + LT - 1) / LT;
    const int64_t tiles = (a.M + LT - 1) / LT * a.tn;
    if (tiles > 0x7FFFFFFF) return SSCATER_E_INVALID_ARG;
    const int per = 16 / size;
    const bool vec = (uintptr_t)x % 16 == 0 && (uintptr_t)weight % 16 == 0 && a.K % per == 0 && a.ldx % per == 0 &&
                     a.ldw % per == 0;
    const dim3 grid((unsigned)tiles), block(256);
    const hipStream_t s = (hipStream_t)stream;
    if (size == 4 && vec) linear_kernel<true, true><<<grid, block, 0, s>>>(a);
    else if (size == 4) linear_kernel<true, false><<<grid, block, 0, s>>>(a);
    else if (vec) linear_kernel<false, true><<<grid, block, 0, s>>>(a);
    else linear_kernel<false, false><<<grid, block, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSCATER_OK : report_hip_error(e);
}
