// Linear layers over rows of cells: y = act(x W^T + b) + r.
//
// W is the first matrix operand and x the second, so a lane holds four
// consecutive output channels of one row; sums are fp32, rounded once.  Four
// kernels, by the number of rows and channels:
//   few rows      linear_rows_kernel: K shared by the wavefronts, no LDS on the way
//                 in (4 x 256 -> 1024 bf16: 2.9 us, a launch and two round trips);
//   some rows     linear_kernel: tiles of 64 x 64, 128 x 128 or 128 x 64 through LDS
//                 (12000 x 1024 -> 256 fp32 with residual 49 us, 127 TFLOP/s; a head of
//                 42 channels over 53568 x 384 bf16 11.6 us, 4.0 TB/s);
//   many, in bf16 linear_big_kernel: persistent tiles of 256 x 128
//                 (214272 x 384 -> 1536, other operands in each call, 367 us, with gelu
//                 431; 8192^3 1140 us, 965 TFLOP/s, 0.6 of a library product's rate).
//
// fp32: a step's values are split in registers into three bf16 planes of 8
// bits each by cutting off (h + m + l is the value exactly, but for bits below
// 2^-133), and six of the nine products are formed.  m is less than 2^-7 and l
// less than 2^-15 of the value, so the others are at most 2^-21 of the product;
// they have its sign, so what is missing leans towards zero.  Six bf16
// instructions take 0.4 of the fp32 kind's time.  An infinity leaves NaN in its
// lower planes: a NaN sum is formed again from the values.
#include <hip/hip_runtime.h>

#include "../../include/sscater.h"
#include "device_common.h"

#include <algorithm>
#include <type_traits>

namespace ssc {

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
    int packed;           // the output's rows lie one behind the other, in one tile, on a 16-byte boundary
    int rvec, yvec;       // residual and output rows may be accessed 16 bytes at a time
};

// What a copy reads where its tile has nothing.
__device__ __attribute__((aligned(16))) uint32_t linear_zero[4];

// z (1 + erf(z / sqrt 2)) / 2 = max(z, 0) - |z| Phi(-|z|), with log2 Phi(-t) as a
// polynomial in t whose largest error of Phi is least (a linear program over 0 <=
// t <= 6; the leading term is negative, so that it goes on falling from there).
// |error of Phi|: 1.7e-8 of the polynomial with these coefficients, 4.9e-8 as
// evaluated in fp32.  At t = 12 it gives 2^-414: minus infinity comes out as zero,
// the limit.  Eleven vector instructions and one exponential; elementwise_maximum
// keeps NaN, in one instruction (a comparison and a choice: four maps' 384 -> 1536
// layer 435 us, against 430).
__device__ __forceinline__ float gelu(float z) {
    const float t = fminf(fabsf(z), 12.f);
    float p = fmaf(-2.77202616e-06f, t, 3.86204774e-05f);
    p = fmaf(p, t, -1.82546341e-04f);
    p = fmaf(p, t, -1.45873099e-04f);
    p = fmaf(p, t, 7.07547553e-03f);
    p = fmaf(p, t, -5.25050312e-02f);
    p = fmaf(p, t, -4.59204912e-01f);
    p = fmaf(p, t, -1.15110576f);
    p = fmaf(p, t, -1.f);
    return fmaf(-t, __builtin_amdgcn_exp2f(p), __builtin_elementwise_maximum(z, 0.f));
}

typedef __attribute__((address_space(3))) float lds_float;

template <int ACT>
using Act = std::integral_constant<int, ACT>;

template <int ACT>
__device__ __forceinline__ float activate(float z) {
    if constexpr (ACT == SSCATER_ACT_RELU) return z < 0.f ? 0.f : z;
    if constexpr (ACT == SSCATER_ACT_GELU) return gelu(z);
    if constexpr (ACT == SSCATER_ACT_SILU)
        return z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * z));
    return z;
}

// N values of one activation, chosen once for all of them.
template <int N>
__device__ __forceinline__ void activate_all(float (&z)[N], int act) {
    if (act == SSCATER_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = activate<SSCATER_ACT_RELU>(z[e]);
    } else if (act == SSCATER_ACT_GELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = activate<SSCATER_ACT_GELU>(z[e]);
    } else if (act == SSCATER_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = activate<SSCATER_ACT_SILU>(z[e]);
    }
}

template <bool F32>
__device__ __forceinline__ float load_value(const void* p, int64_t i) {
    if constexpr (F32) return ((const float*)p)[i];
    return __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16);
}


// Channels k.. of a row that starts at value `at` and may be aligned to its values
// only: 16 bytes, zeros from channel K on.
template <bool F32>
__device__ __forceinline__ uint4 load_piece(const void* base, int64_t at, int k, int K) {
    constexpr int E = F32 ? 4 : 8;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (k + E <= K) {
        __builtin_memcpy(&v, (const char*)base + (at + k) * (F32 ? 4 : 2), 16);
    } else if (k < K) {
        uint32_t b[4] = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (k + e >= K) continue;
            if constexpr (F32) b[e] = ((const uint32_t*)base)[at + k + e];
            else b[e / 2] |= (uint32_t)((const uint16_t*)base)[at + k + e] << (16 * (e & 1));
        }
        v = make_uint4(b[0], b[1], b[2], b[3]);
    }
    return v;
}

// 16-byte piece `piece` of tile row `row` in LDS: rows of RB bytes, the pieces
// of neighbouring rows moved so that lanes which read one piece of eight rows
// fall on different banks.
template <int RB>
__device__ __forceinline__ int place(int row, int piece) {
    if constexpr (RB == 64) return row * 64 + ((piece ^ (row >> 2)) & 3) * 16;
    return row * 128 + ((piece ^ (row >> 1)) & 7) * 16;
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
                v[i] = load_piece<F32>(base, row * ld, k, K);
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
// the wavefronts take them in turn.  A lane's rows and pieces are the same
// in every K step, so their offsets from the tile's first value are formed once,
// in 32 bits (the host sees to it that they fit), and a step only moves the
// uniform base: with the addresses formed anew the vector instructions around
// the copies took longer than the matrix instructions.
template <int ROWS, int P, int WAVES = 4>
struct Copied {
    static constexpr int N = ROWS * P / 64 / WAVES;
    const char* base;
    uint32_t off[N];
    __device__ __forceinline__ void init(const void* p, int64_t ld, int64_t row0, int64_t rows) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        base = (const char*)p + row0 * ld * 2;
        const int most = (int)min((int64_t)ROWS, rows - row0) - 1;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = (i * WAVES + wave) * (64 / P) + lane / P;
            off[i] = (uint32_t)min(row, most) * (uint32_t)(ld * 2) + piece(row) * 16;
        }
    }
    static __device__ __forceinline__ int piece(int row) {
        return ((int)threadIdx.x % P) ^ ((row >> 1) & 7);
    }
    // copy i of the K step from channel k
    __device__ __forceinline__ void one(lds_char* lds, int i, int k, int K) const {
        const int wave = threadIdx.x >> 6;
        const char* from = base + (int64_t)k * 2 + off[i];
        if (k + P * 8 > K) {
            const int row = (i * WAVES + wave) * (64 / P) + (threadIdx.x & 63) / P;
            if (k + piece(row) * 8 >= K) from = (const char*)linear_zero;
        }
        copy16(from, lds + (i * WAVES + wave) * 1024);
    }
    __device__ __forceinline__ void copy(lds_char* lds, int k, int K) const {
#pragma unroll
        for (int i = 0; i < N; ++i) one(lds, i, k, K);
    }
};

// One block of sums on its way out where the tile hangs over an edge or rows may
// not be accessed 16 bytes at a time: the lane's row m, its channels n + 8 g +
// 4 h + 0..3 (g = 0..3), with bias, activation, residual and rounding.
template <bool F32, int ACT>
__device__ __forceinline__ void put_edge(const LinearArgs& a, const f16v& acc, const lds_float* bias, int64_t m, int n,
                                         int h) {
    if (m >= a.M) return;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int c = 8 * (e >> 2) + 4 * h + (e & 3);
        if (n + c >= a.N) continue;
        float z = activate<ACT>(acc[e] + bias[c]);
        if (a.res) z += load_value<F32>(a.res, m * a.ldr + n + c);
        if constexpr (F32) ((float*)a.y)[m * a.ldy + n + c] = z;
        else ((uint16_t*)a.y)[m * a.ldy + n + c] = (uint16_t)bf16_pair(z, z);
    }
}

// 32 rows of NI blocks inside the matrix.  They pass through 32 * RB bytes of LDS
// that are the wavefront's own, so that 4 or 8 lanes store one row's bytes
// together (straight from the sums' layout a store is 32 rows of 32 bytes, which
// the memory path takes at a quarter of its rate), and the residual comes the
// other way through the same place.  bf16: lanes r and r + 32 hold the two halves
// of eight channels and swap halves of two groups first.  PAST: the stores pass by
// the caches, where the output is larger than they are (four maps' 384 -> 1536
// layer 389 -> 344 us: x and W stay in L2).
template <bool F32, int ACT, int NI, bool PAST>
__device__ __forceinline__ void put_rows(const LinearArgs& a, const f16v (&acc)[NI], const lds_float* bias,
                                         lds_char* own, int64_t m, int n) {
    constexpr int S = F32 ? 4 : 2, RB = 32 * NI * S, L = RB / 16, RPI = 64 / L;   // lanes of a row, rows of a store
    const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
    typedef uint32_t u4v __attribute__((ext_vector_type(4)));
    typedef uint32_t u2v __attribute__((ext_vector_type(2)));
    typedef __attribute__((address_space(3))) u4v lds_u4v;
    typedef __attribute__((address_space(3))) u2v lds_u2v;
    if (a.res) {
        const char* from = (const char*)a.res + ((m + lane / L) * a.ldr + n) * S + lane % L * 16;
        u4v v[32 / RPI];
#pragma unroll
        for (int i = 0; i < 32 / RPI; ++i) v[i] = *(const u4v*)(from + (int64_t)i * RPI * a.ldr * S);
#pragma unroll
        for (int i = 0; i < 32 / RPI; ++i) *(lds_u4v*)(own + place<RB>(i * RPI + lane / L, lane % L)) = v[i];
    }
    u4v out[NI][4 * S / 4];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        float z[16];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f4v b = *(const __attribute__((address_space(3))) f4v*)(bias + 32 * i + 8 * g + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) z[4 * g + e] = activate<ACT>(acc[i][4 * g + e] + b[e]);
        }
        if (a.res) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                if constexpr (F32) {
                    const u4v v = *(const lds_u4v*)(own + place<RB>(r, 8 * i + 2 * g + h));
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[4 * g + e] += __uint_as_float(v[e]);
                } else {
                    const u2v v = *(const lds_u2v*)(own + place<RB>(r, 4 * i + g) + 8 * h);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        z[4 * g + e] += __uint_as_float(e & 1 ? v[e / 2] & 0xFFFF0000u : v[e / 2] << 16);
                }
            }
        }
        if constexpr (F32) {
#pragma unroll
            for (int g = 0; g < 4; ++g)
                out[i][g] = u4v{__float_as_uint(z[4 * g]), __float_as_uint(z[4 * g + 1]), __float_as_uint(z[4 * g + 2]),
                                __float_as_uint(z[4 * g + 3])};
        } else {
#pragma unroll
            for (int g = 0; g < 4; g += 2) {
                const auto lo = __builtin_amdgcn_permlane32_swap(bf16_pair(z[4 * g], z[4 * g + 1]),
                                                                 bf16_pair(z[4 * g + 4], z[4 * g + 5]), false, false);
                const auto hi = __builtin_amdgcn_permlane32_swap(bf16_pair(z[4 * g + 2], z[4 * g + 3]),
                                                                 bf16_pair(z[4 * g + 6], z[4 * g + 7]), false, false);
                out[i][g / 2] = u4v{lo[0], hi[0], lo[1], hi[1]};
            }
        }
    }
    // the residual's reads above and these writes are of one wavefront, in order
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int g = 0; g < S; ++g) *(lds_u4v*)(own + place<RB>(r, 2 * S * i + 2 * g + h)) = out[i][g];
    char* to = (char*)a.y + ((m + lane / L) * a.ldy + n) * S + lane % L * 16;
#pragma unroll
    for (int i = 0; i < 32 / RPI; ++i) {
        const u4v v = *(const lds_u4v*)(own + place<RB>(i * RPI + lane / L, lane % L));
        u4v* y = (u4v*)(to + (int64_t)i * RPI * a.ldy * S);
        if constexpr (PAST) __builtin_nontemporal_store(v, y);
        else *y = v;
    }
}

// 32 rows of a matrix of few channels that lie one behind the other (no more than
// the wavefront's 32 * NI channels, y_stride = cout): put together in LDS as they
// lie in memory and stored 16 bytes a lane.  32 * N * S bytes are whole pieces.
template <bool F32, int ACT, int NI>
__device__ __forceinline__ void put_packed(const LinearArgs& a, const f16v (&acc)[NI], const lds_float* bias,
                                           lds_char* own, int64_t m) {
    constexpr int S = F32 ? 4 : 2;
    const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int c = 32 * i + 8 * (e >> 2) + 4 * h + (e & 3);
            if (c >= a.N) continue;
            float z = activate<ACT>(acc[i][e] + bias[c]);
            if (a.res) z += load_value<F32>(a.res, (m + r) * a.ldr + c);
            lds_char* to = own + (r * a.N + c) * S;
            if constexpr (F32) *(__attribute__((address_space(3))) float*)to = z;
            else *(__attribute__((address_space(3))) uint16_t*)to = (uint16_t)bf16_pair(z, z);
        }
    char* y = (char*)a.y + m * a.N * S;
    for (int i = lane; i < 2 * a.N * S; i += 64) *(uint4*)(y + i * 16) = lds16(own + i * 16);
}

// A wavefront's TM x TN blocks; own: 4 KB of LDS that no other wavefront uses.
template <bool F32, int ACT, bool FULL, int TM, int TN, bool PAST>
__device__ __forceinline__ void put_blocks(const LinearArgs& a, const f16v (&acc)[TN][TM], const lds_float* bias,
                                           lds_char* own, int64_t m, int n) {
    const int r = threadIdx.x & 31, h = threadIdx.x >> 5 & 1;
    constexpr int NI = !F32 && TN % 2 == 0 ? 2 : 1;
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
        for (int i = 0; i < TN; i += NI) {
            if constexpr (FULL) {
                f16v z[NI];
#pragma unroll
                for (int c = 0; c < NI; ++c) z[c] = acc[i + c][j];
                put_rows<F32, ACT, NI, PAST>(a, z, bias + 32 * i, own, m + 32 * j, n + 32 * i);
            } else {
#pragma unroll
                for (int c = 0; c < NI; ++c)
                    put_edge<F32, ACT>(a, acc[i + c][j], bias + 32 * (i + c), m + 32 * j + r, n + 32 * (i + c), h);
            }
        }
}

// put(activation, full) with both as types, chosen once for a tile.
template <typename Put>
__device__ __forceinline__ void put_tile(const LinearArgs& a, bool inside, const Put& put) {
    const bool full = inside && a.yvec && (a.rvec || !a.res);
    auto all = [&](auto f) __attribute__((always_inline)) {
        if (a.act == SSCATER_ACT_NONE) put(Act<SSCATER_ACT_NONE>{}, f);
        else if (a.act == SSCATER_ACT_RELU) put(Act<SSCATER_ACT_RELU>{}, f);
        else if (a.act == SSCATER_ACT_GELU) put(Act<SSCATER_ACT_GELU>{}, f);
        else put(Act<SSCATER_ACT_SILU>{}, f);
    };
    if (full) all(std::true_type{});
    else all(std::false_type{});
}

// A wavefront owns TM x TN blocks of 32 rows x 32 output channels, the
// workgroup WM x WN (= 4) wavefronts.
template <bool F32, bool VEC, int WM, int WN, int TM, int TN>
struct LinearShape {
    static constexpr int BM = 32 * WM * TM, BN = 32 * WN * TN;
    static constexpr bool COPY = VEC && !F32;          // straight into LDS
    static constexpr int P = 8;          // 16-byte pieces of a row's K step
    static constexpr int BK = P * (F32 ? 4 : 8);       // 32 or 64 channels
    static constexpr int SX = F32 ? BM * 64 * 3 : BM * 16 * P;
    static constexpr int SW = F32 ? BN * 64 * 3 : BN * 16 * P;
    static constexpr int NST = COPY ? 2 : 1;           // stages in LDS
    static constexpr int LDS = NST * (SX + SW) > 16384 ? NST * (SX + SW) : 16384;
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
    // read after the K loop's barriers
    __shared__ __attribute__((aligned(16))) float bias[C::BN];
    if ((int)threadIdx.x < C::BN)
        bias[threadIdx.x] = a.bias && n0 + (int)threadIdx.x < a.N ? load_value<F32>(a.bias, n0 + threadIdx.x) : 0.f;
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
        Copied<C::BM, C::P> x;
        Copied<C::BN, C::P> w;
        x.init(a.x, a.ldx, m0, a.M);
        w.init(a.w, a.ldw, n0, a.N);
        const int steps = (a.K + C::BK - 1) / C::BK;
        auto issue = [&](int k) __attribute__((always_inline)) {
            lds_char* to = lds + (k & 1) * (C::SX + C::SW);
            x.copy(to, k * C::BK, a.K);
            w.copy(to + C::SX, k * C::BK, a.K);
        };
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
        // the next step is under way in registers beside the products (__syncthreads would wait for it; two or three
        // steps ahead took as long)
        Staged<F32, VEC, C::BM, C::P> x;
        Staged<F32, VEC, C::BN, C::P> w;
        x.load(a.x, a.ldx, m0, a.M, 0, a.K);
        w.load(a.w, a.ldw, n0, a.N, 0, a.K);
        for (int k0 = 0; k0 < a.K; k0 += C::BK) {
            x.store(lds);
            w.store(lds + C::SX);
            lds_barrier();
            if (k0 + C::BK < a.K) {
                x.load(a.x, a.ldx, m0, a.M, k0 + C::BK, a.K);
                w.load(a.w, a.ldw, n0, a.N, k0 + C::BK, a.K);
            }
            multiply(lds, lds + C::SX);
            lds_barrier();
        }
    }

    if constexpr (F32) {
        // an infinity leaves a NaN in its lower planes: such sums are formed again from the values
        bool bad = false;
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) bad |= acc[i][j][e] != acc[i][j][e];
        if (__ballot(bad) != 0) {
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int j = 0; j < TM; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int64_t m = m0 + wm + 32 * j + r;
                        const int n = n0 + wn + 32 * i + 8 * (e >> 2) + 4 * h + (e & 3);
                        if (acc[i][j][e] == acc[i][j][e] || m >= a.M || n >= a.N) continue;
                        float z = 0.f;
                        for (int k = 0; k < a.K; ++k)
                            z = fmaf(load_value<F32>(a.x, m * a.ldx + k), load_value<F32>(a.w, n * a.ldw + k), z);
                        acc[i][j][e] = z;
                    }
        }
    }
    auto put = [&](auto act, auto full) __attribute__((always_inline)) {
        lds_char* own = lds + wave * (C::LDS / 4);
        if constexpr (WN == 1 && !decltype(full)::value) {
            if (a.packed) {
#pragma unroll
                for (int j = 0; j < TM; ++j) {
                    const int64_t m = m0 + wm + 32 * j;
                    f16v z[TN];
#pragma unroll
                    for (int i = 0; i < TN; ++i) z[i] = acc[i][j];
                    if (m + 32 <= a.M) {
                        put_packed<F32, decltype(act)::value, TN>(a, z, (const lds_float*)bias, own, m);
                    } else {
#pragma unroll
                        for (int i = 0; i < TN; ++i)
                            put_edge<F32, decltype(act)::value>(a, z[i], (const lds_float*)bias + 32 * i, m + r, 32 * i, h);
                    }
                }
                return;
            }
        }
        put_blocks<F32, decltype(act)::value, decltype(full)::value, TM, TN, false>(
            a, acc, (const lds_float*)bias + wn, own, m0 + wm, n0 + wn);
    };
    put_tile(a, m0 + C::BM <= a.M && n0 + C::BN <= a.N, put);
}

// Many rows and channels, bf16: persistent workgroups of eight wavefronts, one
// on a compute unit, each with tiles of 256 rows x 128 channels (a wavefront
// 64 x 64) one after the other.  K steps of 64 channels go through three LDS
// stages of 48 KB, copied two steps ahead, and on from the end of one tile into
// the next, so that a tile starts on operands that are there already.
//
// Why: a copy takes about 1100 clocks to arrive, 57 KB have to be under way on a
// compute unit to have its 52 bytes a clock from L2 all the time, and one tile's
// first copies come from HBM; as separate workgroups of 128 x 128 with two
// stages the tiles spent half of their time on their first step and their way
// out.  256 x 128 needs 923 clocks of copies for the 1024 of matrix
// instructions in a step.
//
// The tiles of an XCD are a range with the channels going fastest, so that its
// workgroups' rows meet in its L2.  The stages of the next tile are awaited before
// this one's stores are issued: counted among younger stores they could not be.
struct BigShape {
    static constexpr int BM = 256, BN = 128, P = 8, BK = 64, WAVES = 8;
    static constexpr int SX = BM * 128, SW = BN * 128, STAGE = SX + SW, NST = 3;
};

__global__ __launch_bounds__(512) void linear_big_kernel(LinearArgs a) {
    using C = BigShape;
    __shared__ __attribute__((aligned(1024))) char lds_[C::NST * C::STAGE];
    __shared__ __attribute__((aligned(16))) float bias[2][C::BN];
    lds_char* lds = (lds_char*)lds_;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 31, h = lane >> 5;
    const int wm = wave % 4 * 64, wn = wave / 4 * 64;
    const int first = (int)(blockIdx.x & 7) * a.per_xcd + (int)(blockIdx.x >> 3);
    const int end = min(a.tiles, ((int)(blockIdx.x & 7) + 1) * a.per_xcd), stride = (int)(gridDim.x >> 3);
    const int steps = (a.K + C::BK - 1) / C::BK;
    constexpr int CP = (C::BM + C::BN) * C::P / 64 / C::WAVES;   // copies of a wavefront per stage

    // what is copied next
    Copied<C::BM, C::P, C::WAVES> x;
    Copied<C::BN, C::P, C::WAVES> w;
    int tile = first, at = 0, fill = 0;
    auto begin = [&]() __attribute__((always_inline)) {
        x.init(a.x, a.ldx, (int64_t)(tile / a.tn) * C::BM, a.M);
        w.init(a.w, a.ldw, (int64_t)(tile % a.tn) * C::BN, a.N);
    };
    // the copies of a step in four parts, between its products: all at once they
    // keep the wavefronts from their products until the memory path has taken them
    auto issue = [&](int part) __attribute__((always_inline)) {
        if (tile < end) {
            lds_char* to = lds + fill * C::STAGE;
            x.one(to, part, at * C::BK, a.K);
            if (part < 2) w.one(to + C::SX, part, at * C::BK, a.K);
        }
        if (part == 3) {
            if (tile < end && ++at == steps) {
                at = 0;
                tile += stride;
                if (tile < end) begin();
            }
            fill = fill + 1 == C::NST ? 0 : fill + 1;
        }
    };
    if (first >= end) return;
    begin();
#pragma unroll
    for (int i = 0; i < 8; ++i) issue(i & 3);
    wait_vm<0>();
    // A tile's bias comes with the last step of the tile before: awaited at its start it would wait for that one's
    // stores as well.
    auto bias_of = [&](int t) __attribute__((always_inline)) {
        const int n = t % a.tn * C::BN + threadIdx.x;
        return a.bias && t < end && (int)threadIdx.x < C::BN && n < a.N ? load_value<false>(a.bias, n) : 0.f;
    };
    if ((int)threadIdx.x < C::BN) bias[0][threadIdx.x] = bias_of(first);
    int slot = 0, side = 0;
    for (int t = first; t < end; t += stride, side ^= 1) {
        const int64_t m0 = (int64_t)(t / a.tn) * C::BM;
        const int n0 = t % a.tn * C::BN;
        f16v acc[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = f16v{};
        for (int k = 0; k < steps; ++k) {
            // the first two steps of a tile were awaited before the last one's stores; later ones have one younger stage
            // behind them, or none at the end of the last tile
            if (k >= 2) {
                if (tile < end || k + 1 < steps) wait_vm<CP>();
                else wait_vm<0>();
            }
            lds_barrier();
            const lds_char* X = lds + slot * C::STAGE;
            const lds_char* W = X + C::SX;
            uint4 xv[2][2], wv[2][2];
            auto take = [&](int s) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    xv[s & 1][j] = lds16(X + place<128>(wm + 32 * j + r, 2 * s + h));
                    wv[s & 1][j] = lds16(W + place<128>(wn + 32 * j + r, 2 * s + h));
                }
            };
            take(0);
#pragma unroll
            for (int s = 0; s < C::BK / 16; ++s) {
                if (s < 3) take(s + 1);
                issue(s);
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = mfma32(wv[s & 1][i], xv[s & 1][j], acc[i][j]);
            }
            slot = slot + 1 == C::NST ? 0 : slot + 1;
        }
        const float next = bias_of(t + stride);
        if ((int)threadIdx.x < C::BN) bias[side ^ 1][threadIdx.x] = next;
        wait_vm<0>();
        // the stage read last takes no copies before the next barrier but one
        lds_barrier();
        lds_char* own = lds + (slot == 0 ? C::NST - 1 : slot - 1) * C::STAGE + wave * 4096;
        auto put = [&](auto act, auto full) __attribute__((always_inline)) {
            put_blocks<false, decltype(act)::value, decltype(full)::value, 2, 2, true>(
                a, acc, (const lds_float*)bias[side] + wn, own, m0 + wm, n0 + wn);
        };
        put_tile(a, m0 + C::BM <= a.M && n0 + C::BN <= a.N, put);
    }
}

// Few rows: a workgroup owns 16 T rows x 16 T output channels and its wavefronts
// share K, each with its operands straight from memory, so that a call is one
// round trip and a sum through LDS.  fp32 takes the fp32 matrix instructions.
template <bool F32, bool VEC, int T>
__global__ __launch_bounds__(256) void linear_rows_kernel(LinearArgs a) {
    constexpr int E = F32 ? 4 : 8, BK = 4 * E;         // channels of a lane, and of a wavefront's piece
    __shared__ float sums[4][T * T * 4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n0 = (int)(blockIdx.x % a.tn) * (16 * T);
    const int64_t m0 = (int64_t)(blockIdx.x / a.tn) * (16 * T);
    int64_t xo[T], wo[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        xo[t] = min(m0 + 16 * t + (lane & 15), a.M - 1) * a.ldx;
        wo[t] = min(n0 + 16 * t + (lane & 15), a.N - 1) * a.ldw;
    }
    f4v acc[T][T];                                     // [channels][rows]
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
        for (int j = 0; j < T; ++j) acc[i][j] = f4v{0.f, 0.f, 0.f, 0.f};
    auto load = [&](const void* p, int64_t o, int k) __attribute__((always_inline)) {
        if constexpr (VEC) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (k < a.K) v = *(const uint4*)((const char*)p + (o + k) * (F32 ? 4 : 2));
            return v;
        } else {
            return load_piece<F32>(p, o, k, a.K);
        }
    };
    constexpr int U = VEC ? 4 : 2;                     // pieces in flight
    for (int k0 = wave * BK; k0 < a.K; k0 += 4 * BK * U) {
        uint4 x[U][T], w[U][T];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = k0 + u * 4 * BK + (lane >> 4) * E;
#pragma unroll
            for (int t = 0; t < T; ++t) {
                w[u][t] = load(a.w, wo[t], k);
                x[u][t] = load(a.x, xo[t], k);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < T; ++i)
#pragma unroll
                for (int j = 0; j < T; ++j) {
                    if constexpr (F32) {
                        const uint32_t wv[4] = {w[u][i].x, w[u][i].y, w[u][i].z, w[u][i].w};
                        const uint32_t xv[4] = {x[u][j].x, x[u][j].y, x[u][j].z, x[u][j].w};
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(wv[e]),
                                                                             __uint_as_float(xv[e]), acc[i][j], 0, 0, 0);
                    } else {
                        acc[i][j] = mfma_bf16(w[u][i], x[u][j], acc[i][j]);
                    }
                }
    }
    // lane l, register e: channel 4 (l / 16) + e of row l % 16
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
        for (int j = 0; j < T; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[wave][(i * T + j) * 4 + e][lane] = acc[i][j][e];
    __syncthreads();
    const int c = threadIdx.x & 15, row = threadIdx.x >> 4;
#pragma unroll
    for (int j = 0; j < T; ++j)
#pragma unroll
        for (int i = 0; i < T; ++i) {
            const int n = n0 + 16 * i + c, at = (c >> 2) * 16 + row, e = (i * T + j) * 4 + (c & 3);
            const int64_t m = m0 + 16 * j + row;
            if (n >= a.N || m >= a.M) continue;
            float z[1] = {(sums[0][e][at] + sums[1][e][at]) + (sums[2][e][at] + sums[3][e][at])};
            if (a.bias) z[0] += load_value<F32>(a.bias, n);
            activate_all(z, a.act);
            if (a.res) z[0] += load_value<F32>(a.res, m * a.ldr + n);
            if constexpr (F32) ((float*)a.y)[m * a.ldy + n] = z[0];
            else ((uint16_t*)a.y)[m * a.ldy + n] = (uint16_t)bf16_pair(z[0], z[0]);
        }
}

namespace {

template <bool F32, bool VEC, int WM, int WN, int TM, int TN>
void launch_tiles(LinearArgs& a, hipStream_t s) {
    using C = LinearShape<F32, VEC, WM, WN, TM, TN>;
    a.tn = (a.N + C::BN - 1) / C::BN;
    a.tiles = (int)((a.M + C::BM - 1) / C::BM * a.tn);
    a.per_xcd = (a.tiles + 7) / 8;
    a.packed = a.tn == 1 && a.ldy == a.N && (uintptr_t)a.y % 16 == 0;
    linear_kernel<F32, VEC, WM, WN, TM, TN><<<dim3((unsigned)a.per_xcd * 8), dim3(256), 0, s>>>(a);
}

void launch_big(LinearArgs& a, hipStream_t s) {
    a.tn = (a.N + BigShape::BN - 1) / BigShape::BN;
    a.tiles = (int)((a.M + BigShape::BM - 1) / BigShape::BM * a.tn);
    a.per_xcd = (a.tiles + 7) / 8;
    linear_big_kernel<<<dim3(256), dim3(512), 0, s>>>(a);
}

template <bool F32, bool VEC>
void launch_linear(LinearArgs& a, hipStream_t s) {
    // Which kernel, by how many tiles there are for 256 compute units (us on either side of each bound):
    // fewer than 128 tiles of 64 x 64 leave units idle for all of K, so K is shared (500 x 512 -> 512 fp32, 64 tiles: rows
    // 9.8, tiles 17.0; 600 x 1024 -> 1024 bf16, 160 tiles: rows 13.6, tiles 10.4); the rows kernel's larger block from 512
    // blocks on (64 x 1536 -> 1536, 384 of them: one 7.5, larger 8.3; 128 rows, 768: 10.2 and 8.4)
    const int64_t n16 = (a.N + 15) / 16, n32 = (a.N + 31) / 32;
    if (a.M <= 64 || (a.M + 63) / 64 * ((a.N + 63) / 64) < 128) {
        const int64_t small = (a.M + 15) / 16 * n16;
        const bool one = small <= 512;
        a.tn = (int)(one ? n16 : n32);
        const dim3 grid((unsigned)(one ? small : (a.M + 31) / 32 * n32));
        if (one) linear_rows_kernel<F32, VEC, 1><<<grid, dim3(256), 0, s>>>(a);
        else linear_rows_kernel<F32, VEC, 2><<<grid, dim3(256), 0, s>>>(a);
        return;
    }
    // the persistent kernel where its passes over the card are nearly full (53568 x 384 -> 384, 630 of 768 places: 29.3,
    // tiles of 128 31.9; 24000 x 256 -> 512, 376 of 512: 23.5 and 17.7), a little less so for a long K (8192 x 1536 ->
    // 1536, 384 of 512: 52.2 and 60.2)
    if constexpr (!F32 && VEC) {
        const int64_t tiles = (a.M + BigShape::BM - 1) / BigShape::BM * ((a.N + BigShape::BN - 1) / BigShape::BN);
        const int64_t places = (tiles + 255) / 256 * 256;
        if (a.N > 64 && (tiles * 5 >= places * 4 || (tiles * 10 >= places * 7 && a.K >= 1024))) return launch_big(a, s);
    }
    // a tile of all channels, unless rows of exactly 64 can be stored as they are, once there is one for every compute unit
    // (384 -> 42 bf16: 16384 rows 9.1, tiles of 64 x 64 8.4; 32768: 10.8 and 10.9; 53568: 11.7 and 15.6; 256 -> 42 fp32:
    // 14.1 and 11.1, 14.7 and 13.9, 17.5 and 20.7)
    if (a.N <= 64 && !(a.N == 64 && a.yvec) && a.M >= 256 * 128) return launch_tiles<F32, VEC, 4, 1, 1, 2>(a, s);
    // 128 x 128 from 400 of them on (12000 x 256 -> 512 bf16, 376: 13.4, 64 x 64 10.1; 30000 x 1536 -> 256, 470: 33.2 and
    // 43.8; 12000 x 1024 -> 256 fp32, 188: 63.7 and 50.7)
    if (a.N > 64 && (a.M + 127) / 128 * ((a.N + 127) / 128) >= 400) return launch_tiles<F32, VEC, 2, 2, 2, 2>(a, s);
    return launch_tiles<F32, VEC, 2, 2, 1, 1>(a, s);
}

// Parts of a call that are one launch each: at most 2^22 channels, and rows whose
// smallest tiles (64 x 64) are no more than LAUNCH_GROUPS.  All but the last have
// rows and channels in multiples of 256, so that they keep the call's alignment.
template <bool F32, bool VEC>
void launch_parts(const LinearArgs& all, hipStream_t s) {
    constexpr int64_t SIZE = F32 ? 4 : 2, CHANNELS = 1 << 22;
    const int64_t tn = (std::min((int64_t)all.N, CHANNELS) + 63) / 64, rows = 64 * (LAUNCH_GROUPS / tn & ~int64_t(3));
    for (int64_t n = 0; n < all.N; n += CHANNELS)
        for (int64_t m = 0; m < all.M; m += rows) {
            LinearArgs a = all;
            a.N = (int)std::min(CHANNELS, all.N - n);
            a.M = std::min(rows, all.M - m);
            a.x = (const char*)all.x + m * all.ldx * SIZE;
            a.w = (const char*)all.w + n * all.ldw * SIZE;
            a.bias = all.bias ? (const char*)all.bias + n * SIZE : nullptr;
            a.res = all.res ? (const char*)all.res + (m * all.ldr + n) * SIZE : nullptr;
            a.y = (char*)all.y + (m * all.ldy + n) * SIZE;
            launch_linear<F32, VEC>(a, s);
        }
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
    if (spec->cout > (int64_t(1) << 40) / spec->rows) return SSCATER_E_INVALID_ARG;
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
    // 256 rows of a tile within 32-bit offsets
    const bool vec = (uintptr_t)x % 16 == 0 && (uintptr_t)weight % 16 == 0 && a.K % per == 0 && a.ldx % per == 0 &&
                     a.ldw % per == 0 && std::max(a.ldx, a.ldw) < (1 << 22);
    a.yvec = (uintptr_t)y % 16 == 0 && a.ldy % per == 0;
    a.rvec = (uintptr_t)residual % 16 == 0 && a.ldr % per == 0;
    const hipStream_t s = (hipStream_t)stream;
    if (size == 4) vec ? launch_parts<true, true>(a, s) : launch_parts<true, false>(a, s);
    else vec ? launch_parts<false, true>(a, s) : launch_parts<false, false>(a, s);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSCATER_OK : report_hip_error(e);
}
