// The norms before and after a block, with the gate, the residual scale and the
// residual stream between them:
//
//   t = act(gate) * P(block) * scale,  P(u) = (u - c) / sqrt(mean((u - c)^2) + eps) * w + b
//   sum = x + t,  y = N(sum)           with c the mean or zero, N like P with weights of its own
//
// Every value is read and written once: a row's values stay in the registers of
// the lanes that share it, in fp32, through both norms (a mean first and the
// squares about it afterwards, of values that are there already), and y is formed
// from the sum before that is rounded.
#include "tokens.h"

#include <algorithm>

namespace ssc {

struct NormArgs {
    const void* x;
    const void* block;
    const void* bw;
    const void* bb;
    const void* gate;
    const void* scale;
    const void* w;
    const void* b;
    void* sum;
    void* y;
    int64_t rows, row0;
    int64_t ldx, ldb, ldg, lds, ldy;
    int64_t gate_rows;     // rows that share one of the gate's
    int width, lanes;      // lanes of a row
    int center, act, post;
    float eps;
};

// Values k.. of a row: sixteen bytes of them as fp32, zeros from `width` on.  Rows
// may be aligned to their values only.
template <bool F32, int E>
__device__ __forceinline__ void load_piece(const void* row, int k, int width, float (&v)[E]) {
    uint32_t u[4] = {0, 0, 0, 0};
    if (k + E <= width) {
        __builtin_memcpy(u, (const char*)row + (int64_t)k * (F32 ? 4 : 2), 16);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (k + e < width) {
                if constexpr (F32) u[e] = ((const uint32_t*)row)[k + e];
                else u[e / 2] |= (uint32_t)((const uint16_t*)row)[k + e] << (16 * (e & 1));
            }
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        v[e] = F32 ? __uint_as_float(u[e]) : __uint_as_float(e & 1 ? u[e / 2] & 0xFFFF0000u : u[e / 2] << 16);
}

template <bool F32, int E>
__device__ __forceinline__ void store_piece(void* row, int k, int width, const float (&v)[E]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (F32) u[i] = __float_as_uint(v[i]);
        else u[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
    }
    if (k + E <= width) {
        __builtin_memcpy((char*)row + (int64_t)k * (F32 ? 4 : 2), u, 16);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (k + e < width) {
                if constexpr (F32) ((uint32_t*)row)[k + e] = u[e];
                else ((uint16_t*)row)[k + e] = (uint16_t)(u[e / 2] >> (16 * (e & 1)));
            }
    }
}

__device__ __forceinline__ float gate_value(float g, int act) {
    if (act == SSCATER_ACT_NONE) return g;
    const float s = 1.f / (1.f + expf(-g));
    return act == SSCATER_ACT_SILU ? g * s : s;
}

// A row's sum over its lanes, at most a wavefront of them or the whole workgroup.
__device__ __forceinline__ float row_sum(float v, int lanes, float (&part)[2][4], int& turn) {
    for (int o = 1; o < min(lanes, 64); o <<= 1) v += __shfl_xor(v, o);
    if (lanes > 64) {                                  // uniform: the launch's
        // two sets in turn: the next sum's writers need not wait for this one's readers
        if ((threadIdx.x & 63) == 0) part[turn][threadIdx.x >> 6] = v;
        __syncthreads();
        v = (part[turn][0] + part[turn][1]) + (part[turn][2] + part[turn][3]);
        turn ^= 1;
    }
    return v;
}

// NP pieces of 16 bytes a lane; piece i of lane s of a row is its piece i * lanes + s.
template <bool F32, int NP>
__global__ __launch_bounds__(256) void norm_kernel(NormArgs a) {
    constexpr int S = F32 ? 4 : 2, E = 16 / S;
    __shared__ float part[2][4];
    int turn = 0;
    const int per = 256 / a.lanes, sub = threadIdx.x % a.lanes;
    const int64_t at = a.row0 + (int64_t)blockIdx.x * per + threadIdx.x / a.lanes;
    const int64_t row = min(at, a.rows - 1);           // lanes behind the last row take part in the sums
    auto piece = [&](int i) __attribute__((always_inline)) { return (i * a.lanes + sub) * E; };
    float z[NP][E], x[NP][E], g[NP][E];
    const char* block = (const char*)a.block + row * a.ldb * S;
#pragma unroll
    for (int i = 0; i < NP; ++i) load_piece<F32>(block, piece(i), a.width, z[i]);
    if (a.x) {
#pragma unroll
        for (int i = 0; i < NP; ++i) load_piece<F32>((const char*)a.x + row * a.ldx * S, piece(i), a.width, x[i]);
    }
    if (a.gate) {
        const char* gate = (const char*)a.gate + (a.gate_rows == 1 ? row : row / a.gate_rows) * a.ldg * S;
#pragma unroll
        for (int i = 0; i < NP; ++i) load_piece<F32>(gate, piece(i), a.width, g[i]);
    }
    const float inv = 1.f / a.width;
    auto normed = [&](const void* w, const void* b) __attribute__((always_inline)) {
        if (a.center) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) s += z[i][e];
            const float mean = row_sum(s, a.lanes, part, turn) * inv;
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) z[i][e] = piece(i) + e < a.width ? z[i][e] - mean : 0.f;
        }
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) s = fmaf(z[i][e], z[i][e], s);
        const float r = 1.f / sqrtf(row_sum(s, a.lanes, part, turn) * inv + a.eps);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            float v[E], c[E];
            if (w) load_piece<F32>(w, piece(i), a.width, v);
            if (b) load_piece<F32>(b, piece(i), a.width, c);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                z[i][e] *= r;
                if (w) z[i][e] *= v[e];
                if (b) z[i][e] += c[e];
            }
        }
    };
    if (a.post) normed(a.bw, a.bb);
    if (a.gate) {
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) z[i][e] *= gate_value(g[i][e], a.act);
    }
    if (a.scale) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            float v[E];
            load_piece<F32>(a.scale, piece(i), a.width, v);
#pragma unroll
            for (int e = 0; e < E; ++e) z[i][e] *= v[e];
        }
    }
    if (a.x) {
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) z[i][e] += x[i][e];
    }
    const bool live = at < a.rows;
    if (a.sum && live) {
#pragma unroll
        for (int i = 0; i < NP; ++i) store_piece<F32>((char*)a.sum + row * a.lds * S, piece(i), a.width, z[i]);
    }
    if (!a.y) return;
    // values behind the row's end: the gate and the norm may have left something there
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) z[i][e] = piece(i) + e < a.width ? z[i][e] : 0.f;
    normed(a.w, a.b);
    if (live) {
#pragma unroll
        for (int i = 0; i < NP; ++i) store_piece<F32>((char*)a.y + row * a.ldy * S, piece(i), a.width, z[i]);
    }
}

// Rows of more values than a workgroup's registers hold: they are formed again for
// every sum (from the last-level cache), a workgroup a row.
template <bool F32>
__global__ __launch_bounds__(256) void norm_wide_kernel(NormArgs a) {
    constexpr int S = F32 ? 4 : 2, E = 16 / S;
    __shared__ float part[2][4];
    int turn = 0;
    const int64_t row = a.row0 + blockIdx.x;
    const char* block = (const char*)a.block + row * a.ldb * S;
    const char* res = (const char*)a.x + row * a.ldx * S;
    const char* gate = (const char*)a.gate + row / a.gate_rows * a.ldg * S;
    const float inv = 1.f / a.width;
    float mean = 0.f, r = 1.f;                         // of the block
    auto scaled = [&](float (&z)[E], int k, const void* w, const void* b) __attribute__((always_inline)) {
        float v[E];
        if (w) {
            load_piece<F32>(w, k, a.width, v);
#pragma unroll
            for (int e = 0; e < E; ++e) z[e] *= v[e];
        }
        if (b) {
            load_piece<F32>(b, k, a.width, v);
#pragma unroll
            for (int e = 0; e < E; ++e) z[e] += v[e];
        }
    };
    auto total = [&](float (&z)[E], int k) __attribute__((always_inline)) {
        float v[E];
        load_piece<F32>(block, k, a.width, z);
        if (a.post) {
#pragma unroll
            for (int e = 0; e < E; ++e) z[e] = (z[e] - mean) * r;
            scaled(z, k, a.bw, a.bb);
        }
        if (a.gate) {
            load_piece<F32>(gate, k, a.width, v);
#pragma unroll
            for (int e = 0; e < E; ++e) z[e] *= gate_value(v[e], a.act);
        }
        if (a.scale) scaled(z, k, a.scale, nullptr);
        if (a.x) {
            load_piece<F32>(res, k, a.width, v);
#pragma unroll
            for (int e = 0; e < E; ++e) z[e] += v[e];
        }
    };
    // mean (where it is taken off) and one over the root of what `value` gives
    auto moments = [&](auto value, float& m, float& root) __attribute__((always_inline)) {
        m = 0.f;
        float s = 0.f;
        if (a.center) {
            for (int k = threadIdx.x * E; k < a.width; k += 256 * E) {
                float z[E];
                value(z, k);
#pragma unroll
                for (int e = 0; e < E; ++e) s += k + e < a.width ? z[e] : 0.f;
            }
            m = row_sum(s, 256, part, turn) * inv;
            s = 0.f;
        }
        for (int k = threadIdx.x * E; k < a.width; k += 256 * E) {
            float z[E];
            value(z, k);
#pragma unroll
            for (int e = 0; e < E; ++e) s += k + e < a.width ? (z[e] - m) * (z[e] - m) : 0.f;
        }
        root = 1.f / sqrtf(row_sum(s, 256, part, turn) * inv + a.eps);
    };
    if (a.post) {
        float m, root;
        moments([&](float (&z)[E], int k) __attribute__((always_inline)) { load_piece<F32>(block, k, a.width, z); }, m, root);
        mean = m;
        r = root;
    }
    float m = 0.f, root = 1.f;
    if (a.y) moments(total, m, root);
    for (int k = threadIdx.x * E; k < a.width; k += 256 * E) {
        float z[E];
        total(z, k);
        if (a.sum) store_piece<F32>((char*)a.sum + row * a.lds * S, k, a.width, z);
        if (!a.y) continue;
#pragma unroll
        for (int e = 0; e < E; ++e) z[e] = (z[e] - m) * root;
        scaled(z, k, a.w, a.b);
        store_piece<F32>((char*)a.y + row * a.ldy * S, k, a.width, z);
    }
}

namespace {

constexpr int NORM_PIECES = 4;                         // at most of a lane

template <bool F32>
void launch_norm(NormArgs a, hipStream_t s) {
    const int pieces = (a.width + (F32 ? 3 : 7)) / (F32 ? 4 : 8);
    int np = 0;
    a.lanes = 256;
    if (pieces <= 64 * NORM_PIECES) {
        // the lanes that leave the fewest places without a piece, of those the most
        int best = 1 << 30;
        for (int l = 1; l <= 64; l <<= 1) {
            const int n = (pieces + l - 1) / l;
            if (n <= NORM_PIECES && n * l <= best) {
                best = n * l;
                a.lanes = l;
                np = n;
            }
        }
    } else if (pieces <= 256 * NORM_PIECES) {
        np = (pieces + 255) / 256;
    }
    const int per = np ? 256 / a.lanes : 1;
    for (int64_t row = 0; row < a.rows; row += LAUNCH_GROUPS * per) {
        a.row0 = row;
        const dim3 grid((unsigned)std::min(LAUNCH_GROUPS, (a.rows - row + per - 1) / per)), block(256);
        if (np == 0) norm_wide_kernel<F32><<<grid, block, 0, s>>>(a);
        else if (np == 1) norm_kernel<F32, 1><<<grid, block, 0, s>>>(a);
        else if (np == 2) norm_kernel<F32, 2><<<grid, block, 0, s>>>(a);
        else if (np == 3) norm_kernel<F32, 3><<<grid, block, 0, s>>>(a);
        else norm_kernel<F32, 4><<<grid, block, 0, s>>>(a);
    }
}

}  // namespace

}  // namespace ssc

using namespace ssc;

extern "C" int sscater_norm(const sscater_norm_spec* spec, const void* x, const void* block, const void* block_weight,
                            const void* block_bias, const void* gate, const void* scale, const void* weight,
                            const void* bias, void* sum, void* y, void* stream) {
    if (!spec || (spec->dtype != SSCATER_F32 && spec->dtype != SSCATER_BF16)) return SSCATER_E_INVALID_ARG;
    const int64_t C = spec->width, rows = spec->rows;
    if (rows < 0 || rows > (int64_t(1) << 36) || C < 1 || C > (1 << 30) || rows * C > (int64_t(1) << 40))
        return SSCATER_E_INVALID_ARG;
    if (spec->center < 0 || spec->center > 1 || spec->block_norm < 0 || spec->block_norm > 1 || !(spec->eps >= 0.f) ||
        (spec->activation != SSCATER_ACT_NONE && spec->activation != SSCATER_ACT_SILU &&
         spec->activation != SSCATER_ACT_SIGMOID))
        return SSCATER_E_INVALID_ARG;
    if (rows == 0) return SSCATER_OK;
    if ((!spec->block_norm && (block_weight || block_bias)) || (!y && (weight || bias)) || (!sum && !y))
        return SSCATER_E_INVALID_ARG;
    if (spec->block_stride < C || (x && spec->x_stride < C) || (gate && spec->gate_stride < C) ||
        (sum && spec->sum_stride < C) || (y && spec->y_stride < C))
        return SSCATER_E_INVALID_ARG;
    if (gate && (spec->gate_rows < 1 || rows % spec->gate_rows)) return SSCATER_E_INVALID_ARG;
    const int size = spec->dtype == SSCATER_F32 ? 4 : 2;
    for (const void* p : {x, block, block_weight, block_bias, gate, scale, weight, bias, (const void*)sum, (const void*)y})
        if ((uintptr_t)p % size) return SSCATER_E_INVALID_ARG;
    if (!block) return SSCATER_E_INVALID_ARG;
    NormArgs a;
    a.x = x; a.block = block; a.bw = block_weight; a.bb = block_bias; a.gate = gate; a.scale = scale; a.w = weight;
    a.b = bias; a.sum = sum; a.y = y;
    a.rows = rows; a.row0 = 0;
    a.ldx = spec->x_stride; a.ldb = spec->block_stride; a.ldg = spec->gate_stride; a.lds = spec->sum_stride;
    a.ldy = spec->y_stride;
    a.gate_rows = gate ? spec->gate_rows : 1;
    a.width = (int)C; a.center = spec->center; a.act = spec->activation; a.post = spec->block_norm; a.eps = spec->eps;
    if (spec->dtype == SSCATER_F32) launch_norm<true>(a, (hipStream_t)stream);
    else launch_norm<false>(a, (hipStream_t)stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSCATER_OK : report_hip_error(e);
}
