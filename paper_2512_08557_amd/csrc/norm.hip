// The norms before and after a block, with the gate, the residual scale and the
// residual stream between them:
//
//   t = act(gate) * P(block) * scale,  P(u) = (u - c) / sqrt(mean((u - c)^2) + eps) * w + b
//   sum = x + t,  y = N(sum)           with c the mean or zero, N like P with weights of its own
//
// Every value is read and written once: a row's values stay in the registers of
// the lanes that share it, in fp32, through both norms (a mean first and the
// squares about it afterwards, of values that are there already), and y is formed
// from the sum before that is rounded.  Those lanes take several rows, the next
// one's values under way while this one's are worked on; what the rows share
// (weights, an image's gate times the scale) stays in registers too.
//
// Bound by memory: 214272 rows of 384 bf16 values (norm, image gates, residual, norm:
// 658 MB) 141 us, 4.7 TB/s where a large copy has 4.7 to 5.1; of fp32 262 us, 5.0; the
// norm alone 70 and 127.  20000 rows through both norms, less their means: 2048 values
// 77 us in bf16 and 131 in fp32 (4.3 and 5.0 TB/s), 4096 141 and 260 (4.6, 5.0).  Wider
// ones see below.
#include "tokens.h"

#include <algorithm>
#include <type_traits>

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
    int each;              // rows of the same lanes
    int whole;             // all their pieces are there
    int center, act, post;
    float eps;
};

// Sixteen bytes of a row, values k .. of it, and zeros from `width` on.  Rows may be aligned to their values only.
template <bool F32>
__device__ __forceinline__ uint4 load_raw(const void* row, int k, int width) {
    constexpr int E = F32 ? 4 : 8;
    uint32_t u[4] = {0, 0, 0, 0};
    if (k + E <= width) {
        __builtin_memcpy(u, (const char*)row + (int64_t)k * (F32 ? 4 : 2), 16);
    } else if (k < width) {
        // the row's end: eight bytes, four, two, as many as there are
        const int n = (width - k) * (F32 ? 4 : 2);
        const char* at = (const char*)row + (int64_t)k * (F32 ? 4 : 2);
        uint32_t w = 0;
        if (n & 8) __builtin_memcpy(u, at, 8);
        if (n & 4) __builtin_memcpy(&w, at + (n & 8), 4);
        if ((n & 12) == 12) u[2] = w;
        else if (n & 4) u[0] = w;
        if constexpr (!F32) {
            uint16_t h = 0;
            if (n & 2) __builtin_memcpy(&h, at + (n & 12), 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = (n & 2) && n / 4 == i ? h : u[i];
        }
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}

template <bool F32, int E>
__device__ __forceinline__ void unpack(const uint4 raw, float (&v)[E]) {
    const uint32_t u[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int e = 0; e < E; ++e)
        v[e] = F32 ? __uint_as_float(u[e]) : __uint_as_float(e & 1 ? u[e / 2] & 0xFFFF0000u : u[e / 2] << 16);
}

template <bool F32, int E>
__device__ __forceinline__ void load_piece(const void* row, int k, int width, float (&v)[E]) {
    unpack<F32>(load_raw<F32>(row, k, width), v);
}

template <bool F32, int E>
__device__ __forceinline__ void store_piece(void* row, int k, int width, const float (&v)[E]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (F32) u[i] = __float_as_uint(v[i]);
        else u[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
    }
    char* const at = (char*)row + (int64_t)k * (F32 ? 4 : 2);
    if (k + E <= width) {
        __builtin_memcpy(at, u, 16);
    } else if (k < width) {
        const int n = (width - k) * (F32 ? 4 : 2);
        if (n & 8) __builtin_memcpy(at, u, 8);
        if (n & 4) {
            const uint32_t w = n & 8 ? u[2] : u[0];
            __builtin_memcpy(at + (n & 8), &w, 4);
        }
        if constexpr (!F32)
            if (n & 2) {
                const uint16_t h = (uint16_t)(n & 8 ? n & 4 ? u[3] : u[2] : n & 4 ? u[1] : u[0]);
                __builtin_memcpy(at + (n & 12), &h, 2);
            }
    }
}

// The exponential is of the product with log2(e) and, to first order, of that product's rounding: at -80 the rounding
// alone would be 4e-6 of the result.
__device__ __forceinline__ float gate_value(float g, int act) {
    if (act == SSCATER_ACT_NONE) return g;
    const float t = -1.44269504f * g, low = fmaf(-1.44269504f, g, -t) - 1.92596303e-8f * g, x = __builtin_amdgcn_exp2f(t);
    const float s = __builtin_amdgcn_rcpf(1.f + (fabsf(t) < 126.f ? fmaf(x, 0.69314718f * low, x) : x));
    return act == SSCATER_ACT_SILU ? g * s : s;
}

// A row's sum over its lanes, at most a wavefront of them or the whole workgroup; the same bits in all.
__device__ __forceinline__ float row_sum(float v, int lanes, float (&part)[2][4], int& turn) {
    auto add = [&](auto ctrl) __attribute__((always_inline)) {
        constexpr int C = decltype(ctrl)::value;
        v += __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), C, 0xF, 0xF, true));
    };
    if (lanes > 1) add(std::integral_constant<int, 0xB1>{});       // the neighbour
    if (lanes > 2) add(std::integral_constant<int, 0x4E>{});       // the other pair of four
    if (lanes > 4) add(std::integral_constant<int, 0x141>{});      // the other four of eight, back to front
    if (lanes > 8) add(std::integral_constant<int, 0x140>{});      // the other eight of sixteen, the same
    if (lanes > 16) v += __shfl_xor(v, 16);
    if (lanes > 32) v += __shfl_xor(v, 32);
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
// Registers for two wavefronts a SIMD (NP = 1: four); the compiler left alone takes 261 for three pieces of bf16, and one
// wavefront a SIMD is 254 us over four maps for 150.  With two, three pieces of bf16 spill four registers, and four pieces
// 73: 20000 rows of 6144 values go through both norms in 198 us (5.0 TB/s), of 8192 in 506 (2.6).
template <bool F32, int NP>
__global__ __launch_bounds__(256, (NP == 1 ? 4 : 2)) void norm_kernel(NormArgs a) {
    constexpr int S = F32 ? 4 : 2, E = 16 / S;
    __shared__ float part[2][4];
    int turn = 0;
    const int per = 256 / a.lanes, sub = threadIdx.x % a.lanes;
    const int64_t first = a.row0 + ((int64_t)blockIdx.x * per + threadIdx.x / a.lanes) * a.each;
    auto piece = [&](int i) __attribute__((always_inline)) { return (i * a.lanes + sub) * E; };
    uint4 w[NP], b[NP], bw[NP], bb[NP];
    float gs[NP][E];                                   // act(gate) * scale
    auto vector = [&](const void* v, uint4 (&to)[NP]) __attribute__((always_inline)) {
        if (v)
#pragma unroll
            for (int i = 0; i < NP; ++i) to[i] = load_raw<F32>(v, piece(i), a.width);
    };
    vector(a.w, w);
    vector(a.b, b);
    vector(a.bw, bw);
    vector(a.bb, bb);
    struct Row {
        uint4 x[NP], z[NP];
    };
    // lanes behind the last row take part in the sums
    auto load = [&](int64_t at, Row& r) __attribute__((always_inline)) {
        const int64_t row = min(at, a.rows - 1);
#pragma unroll
        for (int i = 0; i < NP; ++i) r.z[i] = load_raw<F32>((const char*)a.block + row * a.ldb * S, piece(i), a.width);
        if (a.x) {
#pragma unroll
            for (int i = 0; i < NP; ++i) r.x[i] = load_raw<F32>((const char*)a.x + row * a.ldx * S, piece(i), a.width);
        }
    };
    auto factors = [&](int64_t row) __attribute__((always_inline)) {
        uint4 g[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) g[i] = load_raw<F32>((const char*)a.gate + row * a.ldg * S, piece(i), a.width);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            unpack<F32>(g[i], gs[i]);
#pragma unroll
            for (int e = 0; e < E; ++e) gs[i][e] = gate_value(gs[i][e], a.act);
            if (a.scale) {
                float v[E];
                load_piece<F32>(a.scale, piece(i), a.width, v);
#pragma unroll
                for (int e = 0; e < E; ++e) gs[i][e] *= v[e];
            }
        }
    };
    // rows left of the gate's row, and that row
    int64_t shared = 0, left = a.rows;
    if (a.gate) {
        if (a.gate_rows > 1) {
            const int64_t row = min(first, a.rows - 1);
            shared = row >> 32 || a.gate_rows >> 32 ? row / a.gate_rows : (uint32_t)row / (uint32_t)a.gate_rows;
            left = (shared + 1) * a.gate_rows - row;
        }
    } else if (a.scale) {
#pragma unroll
        for (int i = 0; i < NP; ++i) load_piece<F32>(a.scale, piece(i), a.width, gs[i]);
    }
    const float inv = 1.f / a.width;
    float z[NP][E];
    auto normed = [&](const void* wp, const uint4 (&wv)[NP], const void* bp, const uint4 (&bv)[NP]) __attribute__((always_inline)) {
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
                for (int e = 0; e < E; ++e) z[i][e] -= mean;
            if (!a.whole) {
#pragma unroll
                for (int i = 0; i < NP; ++i)
#pragma unroll
                    for (int e = 0; e < E; ++e) z[i][e] = piece(i) + e < a.width ? z[i][e] : 0.f;
            }
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
            if (wp) unpack<F32>(wv[i], v);
            if (bp) unpack<F32>(bv[i], c);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                z[i][e] *= r;
                if (wp) z[i][e] *= v[e];
                if (bp) z[i][e] += c[e];
            }
        }
    };
    Row next;
    load(first, next);
    for (int i0 = 0; i0 < a.each; ++i0) {
        const int64_t at = first + i0;
        const Row r = next;
        if (i0 + 1 < a.each) load(at + 1, next);
        if (a.gate) {
            if (a.gate_rows == 1) {
                factors(min(at, a.rows - 1));
            } else if (i0 == 0 || left == 0) {
                if (i0 > 0 && at < a.rows) ++shared;
                if (i0 > 0) left = a.gate_rows;
                factors(shared);
            }
            --left;
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) unpack<F32>(r.z[i], z[i]);
        if (a.post) normed(a.bw, bw, a.bb, bb);
        if (a.gate || a.scale) {
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) z[i][e] *= gs[i][e];
        }
        if (a.x) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                float v[E];
                unpack<F32>(r.x[i], v);
#pragma unroll
                for (int e = 0; e < E; ++e) z[i][e] += v[e];
            }
        }
        const bool live = at < a.rows;
        if (a.sum && live) {
#pragma unroll
            for (int i = 0; i < NP; ++i) store_piece<F32>((char*)a.sum + at * a.lds * S, piece(i), a.width, z[i]);
        }
        if (!a.y) continue;
        if (!a.whole) {                                // the norm's bias may have left something behind the row's end
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) z[i][e] = piece(i) + e < a.width ? z[i][e] : 0.f;
        }
        normed(a.w, w, a.b, b);
        if (live) {
#pragma unroll
            for (int i = 0; i < NP; ++i) store_piece<F32>((char*)a.y + at * a.ldy * S, piece(i), a.width, z[i]);
        }
    }
}

// Rows of more values than a workgroup's registers hold: they are formed again for
// every sum (from the last-level cache), a workgroup a row (20000 fp32 rows of 8192
// values through both norms 892 us, 2.9 TB/s of the bytes that they have; the norm alone
// 313, 4.2; 5000 rows of 20000 690 and 233).
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

// Pieces of a lane: three and the rest of the lane's registers is what a wavefront has where a SIMD holds two (rows of
// 2048 bf16 values, 20000 of them, by four pieces 192 us, by one of a workgroup's lanes 69).
constexpr int NORM_PIECES = 3, NORM_PIECES_GROUP = 4;

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
    } else if (pieces <= 256 * NORM_PIECES_GROUP) {
        np = (pieces + 255) / 256;
    }
    a.whole = np * a.lanes * (F32 ? 4 : 8) == a.width;
    // rows of the same lanes, where there are eight wavefronts for each SIMD (four maps: each for itself 243 us, three
    // 166, eight 147, sixteen 171)
    a.each = np ? (int)std::min((int64_t)8, std::max((int64_t)1, a.rows * a.lanes / 64 / 4096)) : 1;
    const int per = np ? 256 / a.lanes * a.each : 1;
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
    // (the quotient: a product of both limits would pass 64 bits)
    if (rows < 0 || rows > (int64_t(1) << 36) || C < 1 || C > (1 << 30) || (rows > 0 && C > (int64_t(1) << 40) / rows))
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
