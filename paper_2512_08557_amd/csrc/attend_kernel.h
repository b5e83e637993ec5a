// Attention over the token cache (a sliding window and the first tokens of the
// stream), and of queries to the keys of another set of tokens.
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
// with the transposing read (bf16).  exp is taken to base 2, sums in fp32.
//
// The product with bf16 values takes the probabilities in bf16.  Up to 32 rows
// of a key head are bound by the cache's bytes and take them in two parts, which
// hold 16 bits (one token of sixteen streams over 65536 keys 358 us, with one part
// 358; eight tokens over 16384 keys 27.5, 26.9): the error is that of the output's
// rounding alone.  More rows are bound by the products.  Of the cache they take one
// part, an error as large as the output's rounding (a window of 33480 tokens 1920
// us, in two parts 2680; 48 rows over 16384 keys 30.9 and 33.1); of another set of
// tokens two, and one where the caller asks for it (900 queries of four maps of
// 53568 cells, 16 heads of 64 on 4: 1370 us, in one part 980; 8 heads of 32, a
// quarter of the cells visible: 161 and 117; 500 queries over two times 20000 keys,
// 8 heads of 128 on 4: 126 and 96).  The sum is of the unrounded probabilities.
//
// WM of the four wavefronts share keys and take different rows, the other
// 4 / WM groups take other tiles of keys and are joined at the end.  Where the
// rows leave compute units idle the keys are also split over workgroups, whose
// unnormalised sums are joined by a second launch.
#pragma once

#include "tokens.h"

#include <algorithm>
#include <type_traits>

namespace ssc {

typedef short s4v __attribute__((ext_vector_type(4)));

// Where a sequence's keys are: the token cache's slots; rows one behind the other;
// or those rows of them that a list names (the visible ones).
enum class Keys { CACHE, ROWS, LISTED };

struct AttendArgs {
    TokenRows rows;        // of the queries
    const void* q;
    const void* k;
    const void* v;
    void* out;
    float* part;           // [splits][tokens * q_heads][D] unnormalised sums, then [..][2] maximum and sum
    int q_heads, kv_heads, group;
    int sinks, capacity, window, causal;
    int qtiles, splits;
    int id0;               // first workgroup of the launch
    float scale;           // its size times log2(e)
    uint32_t flip;         // sign bits of the queries, flipped for a negative scale
    // ROWS and LISTED: bytes from row to row, the sequences' rows, and the visible ones' numbers within their sequence
    // and how many they are
    int64_t pitch_q;
    uint32_t pitch_k, pitch_v;
    int keys, max_k;
    const int32_t* k_start;
    const int32_t* list;
    const int32_t* count;
};

// Two probabilities in two bf16 parts each: the first 8 bits, and what is left rounded to 8, off by 2^-16 of them.  The
// second part of one that is not zero is not either, nor negative (a 2^-23rd of it is added): an infinite value times both
// is that infinity, not NaN.
__device__ __forceinline__ void two_parts(float x, float y, uint32_t& first, uint32_t& second) {
    constexpr float MORE = 1.f + 0x1p-23f;
    const uint32_t ux = __float_as_uint(x), uy = __float_as_uint(y);
    first = __builtin_amdgcn_perm(uy, ux, 0x07060302u);
    second = bf16_pair(fmaf(x, MORE, -__uint_as_float(ux & 0xFFFF0000u)), fmaf(y, MORE, -__uint_as_float(uy & 0xFFFF0000u)));
}

template <bool F32, int D, int WM>
struct AttendShape {
    static constexpr int S = F32 ? 4 : 2;
    static constexpr int RB = D * S;               // bytes of a cache row
    // fp32 with many rows: keys, values, queries and probabilities as three bf16
    // planes and six of the nine products (as in the linear layers).  K and V are
    // split once per workgroup on their way into LDS, through registers.
    static constexpr bool PL = F32 && WM == 4;
    static constexpr int NP = PL ? 3 : 1;          // planes
    static constexpr int LRB = PL ? D * 2 : RB;    // bytes of a row in LDS
    static constexpr int CPR = LRB / 16;           // its 16-byte pieces
    static constexpr bool B16 = !F32 || PL;        // bf16 operands
    static constexpr int BN = PL ? (D == 32 ? 64 : 32) : F32 || WM == 1 ? 32 : 64;   // keys of a tile
    static constexpr int NT = BN / 32;
    static constexpr int PB = BN * LRB;            // bytes of a plane
    static constexpr int TB = NP * PB;             // bytes of a tile
    static constexpr int NG = BN * RB / 16 / 256;  // pieces of a tile that a thread splits (PL)
    static constexpr int WK = 4 / WM;              // groups over keys
    static constexpr int BM = 32 * WM;
    static constexpr int QN = LRB / 32;            // 16-byte pieces of a lane's half of a query row, of each plane
    static constexpr int ON = D / 2;               // output values of a lane
    static constexpr int GROUP = 4 * TB;           // two tiles of keys and two of values
    static constexpr int LDS = WK * GROUP > 4 * ON * 256 || WK == 1 ? WK * GROUP : 4 * ON * 256;
    static constexpr int WGS = LDS > 80 * 1024 || (F32 && D >= 64) ? 1 : 2;   // workgroups of a compute unit
    static constexpr int RPC = 1024 / LRB;         // rows of a copy
    static constexpr int NC = TB / 1024 / WM;      // copies of a wavefront for a tile of keys, and of values
    // Piece c of row r sits at piece c ^ swap: sixteen lanes that read one piece
    // of neighbouring rows (K), and the four rows of a transposed read by 32 lanes
    // (V, four pieces each), fall on different banks of the 64.  fp32 values are
    // read by 32 lanes from one row and by 32 from the row four further on.
    static __device__ __forceinline__ int swap_k(int r) {
        return CPR == 4 ? (r >> 2) & 3 : CPR == 8 ? (r >> 1) & 7 : r & 15;
    }
    static __device__ __forceinline__ int swap_v(int r) {
        if (!B16) return CPR == 8 ? 0 : (r & 4) * 2;
        return CPR == 4 ? 0 : CPR == 8 ? (r & 2) * 2 : (r & 3) * 4;
    }
};

// What a copy reads for a group without a tile.
static __device__ __attribute__((aligned(16))) uint32_t attend_zero[4];

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

// Whether one of four values is infinite or NaN.
__device__ __forceinline__ bool special(const uint4 v) {
    const uint32_t m = 0x7F800000u;
    return (v.x & m) == m || (v.y & m) == m || (v.z & m) == m || (v.w & m) == m;
}

// Eight values, signs flipped by `flip`, as operands of the three planes.
__device__ __forceinline__ void split8(const uint4 lo, const uint4 hi, uint32_t flip, uint4 (&f)[3], bool& bad) {
    bad |= special(lo) || special(hi);
    cut_pair(lo.x ^ flip, lo.y ^ flip, f[0].x, f[1].x, f[2].x);
    cut_pair(lo.z ^ flip, lo.w ^ flip, f[0].y, f[1].y, f[2].y);
    cut_pair(hi.x ^ flip, hi.y ^ flip, f[0].z, f[1].z, f[2].z);
    cut_pair(hi.z ^ flip, hi.w ^ flip, f[0].w, f[1].w, f[2].w);
}

// The six products of two operands in planes, the small ones first.
__device__ __forceinline__ f16v mfma_planes(const uint4 (&x)[3], const uint4 (&y)[3], f16v c) {
    c = mfma32(x[2], y[0], c);
    c = mfma32(x[0], y[2], c);
    c = mfma32(x[1], y[1], c);
    c = mfma32(x[1], y[0], c);
    c = mfma32(x[0], y[1], c);
    return mfma32(x[0], y[0], c);
}

// ONE: bf16 probabilities in one part, whatever the rows
template <bool F32, int D, int WM, Keys SRC, bool ONE>
__global__ __launch_bounds__(256, (AttendShape<F32, D, WM>::WGS)) void attend_kernel(AttendArgs a) {
    using C = AttendShape<F32, D, WM>;
    constexpr bool CACHE = SRC == Keys::CACHE, LISTED = SRC == Keys::LISTED;
    constexpr int PP = C::PL ? 3 : F32 || ONE ? 1 : 2;   // parts of a probability
    __shared__ __attribute__((aligned(1024))) char lds[C::LDS];
    __shared__ float ml[4][32][2];
    // LISTED: the rows of each group's tiles j + 1 .. j + 3 (and j), copied as the tiles are
    __shared__ __attribute__((aligned(256))) int named[LISTED ? C::WK : 1][4][C::BN];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wk = wave / WM;
    const int h = lane >> 5, col = lane & 31;
    // Key heads go fastest, so that an XCD (workgroup id mod 8) keeps to one or a few of them and finds their keys in
    // its L2; the last tokens' tiles, which reach furthest, come first, and short ones fill up the end.  Of few rows
    // nothing is read twice: there splits go fastest, and every XCD has a part of each sequence, long or short (nine
    // streams of different lengths over up to 65536 keys 190 us, with key heads fastest 215).
    int id = a.id0 + (int)blockIdx.x, kvh, b, split, tile;
    if constexpr (WM == 1) {
        split = id % a.splits;
        id /= a.splits;
        tile = 0;
        kvh = id % a.kv_heads;
        b = id / a.kv_heads;
    } else {
        kvh = id % a.kv_heads;
        id /= a.kv_heads;
        b = id % a.rows.batch;
        id /= a.rows.batch;
        split = id % a.splits;
        tile = a.qtiles - 1 - id / a.splits;
    }
    int first, n;
    rows_of(a.rows, b, first, n);
    const int nr = n * a.group;                    // rows of this key head
    if (tile * C::BM >= nr) return;
    const int64_t past = CACHE ? past_of(a.rows, b) : 0;
    Reach reach;
    int k_first = 0, k_last = 0;                   // ROWS, LISTED: the sequence's first row, and its last from there
    if constexpr (CACHE) {
        const int i0 = tile * C::BM / a.group, i1 = (min((tile + 1) * C::BM, nr) - 1) / a.group;
        reach.lo = max((int64_t)0, (a.causal ? past + i0 : past) - a.window + 1);
        reach.n_sinks = (int)min((int64_t)a.sinks, reach.lo);
        reach.total = (int)min((int64_t)a.capacity,
                               reach.n_sinks + (a.causal ? past + i1 + 1 : past + n) - reach.lo);
        // (a 64-bit remainder takes half a microsecond; streams are that long only after hours)
        const int64_t beyond = max(reach.lo, (int64_t)a.sinks) - a.sinks;
        const uint32_t ring = a.capacity - a.sinks;
        reach.base = beyond >> 32 == 0 ? (int)((uint32_t)beyond % ring) : (int)(beyond % ring);
    } else {
        int kn;
        rows_of(TokenRows{a.keys, a.max_k, a.rows.batch, a.k_start, nullptr}, b, k_first, kn);
        reach.total = LISTED ? min(a.count[b], kn) : kn;
        k_last = kn - 1;
    }
    const int row = min(tile * C::BM + wm * 32 + col, nr - 1);
    const int tok = row / a.group;
    const int64_t qrow = ((int64_t)(first + tok) * a.q_heads + kvh * a.group + row % a.group);
    // the row sees u <= last, and of those u >= from or u < sinks
    int last = reach.total - 1, from = 0;
    if constexpr (CACHE) {
        last = (int)min((int64_t)last, reach.n_sinks + (a.causal ? past + tok : past + n - 1) - reach.lo);
        from = (int)max((int64_t)0, reach.n_sinks + (a.causal ? past + tok : past) - a.window + 1 - reach.lo);
    }

    const char* query = (const char*)a.q + (CACHE ? qrow * C::RB : (first + tok) * a.pitch_q +
                                                                       (kvh * a.group + row % a.group) * C::RB);
    bool again = false;                            // infinities or NaN: see the end of the tiles
    uint4 qf[C::QN][C::NP];
    if constexpr (C::PL) {
        const char* p = query + h * 32;
        bool bad = false;
#pragma unroll
        for (int s = 0; s < C::QN; ++s) {
            const uint4 lo = *(const uint4*)(p + s * 64), hi = *(const uint4*)(p + s * 64 + 16);
            split8(lo, hi, a.flip, qf[s], bad);
        }
        again = __ballot(bad) != 0;
    } else {
        const char* p = query + h * 16;
#pragma unroll
        for (int s = 0; s < C::QN; ++s) {
            qf[s][0] = *(const uint4*)(p + s * 32);
            qf[s][0].x ^= a.flip;
            qf[s][0].y ^= a.flip;
            qf[s][0].z ^= a.flip;
            qf[s][0].w ^= a.flip;
        }
    }
    f16v o[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t) o[t] = f16v{};
    float m = -INFINITY, l = 0.f;

    const int tiles = (reach.total + C::BN - 1) / C::BN;
    const int per = (tiles + a.splits - 1) / a.splits;
    const int tb = min(tiles, split * per), te = min(tiles, tb + per);
    const uint32_t pitch_k = CACHE ? C::RB : a.pitch_k, pitch_v = CACHE ? C::RB : a.pitch_v;
    const int64_t head = CACHE ? ((int64_t)b * a.kv_heads + kvh) * a.capacity * C::RB : kvh * C::RB;
    const char* kg = (const char*)a.k + head + (CACHE ? 0 : (int64_t)k_first * pitch_k);
    const char* vg = (const char*)a.v + head + (CACHE ? 0 : (int64_t)k_first * pitch_v);
    lds_char* own = (lds_char*)lds + wk * C::GROUP;
    // rows of the wavefront that see least, for the choice of the masked form
    const int wl_first = __builtin_amdgcn_readfirstlane(last);
    const int wf_last = __builtin_amdgcn_readlane(from, 31);

    // the group's tiles are tb + wk, tb + wk + WK, ...; groups that share a workgroup go round as often as the first
    const int mine = te - tb > wk ? (te - tb - wk + C::WK - 1) / C::WK : 0;
    const int rounds = WM == 1 ? mine : (te - tb + C::WK - 1) / C::WK;
    auto tile_of = [&](int j) __attribute__((always_inline)) { return tb + wk + j * C::WK; };
    // Copies of a tile: a lane's place within it is always the same, so for keys
    // that lie one behind the other only the uniform base moves.
    const int row0 = wm * C::RPC + lane / C::CPR, pc = lane % C::CPR;
    // Whether tile t's keys lie one behind the other, from cache row `row` on: not
    // where the ring's end, the sinks' end or the last key cuts it.
    auto whole = [&](int t, int& row) __attribute__((always_inline)) {
        const int u = t * C::BN, ring = a.capacity - a.sinks;
        if constexpr (!CACHE) {
            row = u;
            return !LISTED && u + C::BN <= reach.total;
        }
        int x = reach.base + (u - a.sinks);
        if (x >= ring) x -= ring;
        const bool sink = u + C::BN <= a.sinks;
        row = sink ? u : a.sinks + x;
        return u + C::BN <= reach.total && (sink || (u >= a.sinks && x + C::BN <= ring));
    };
    // the rows of the group's round j
    auto name = [&](int j) __attribute__((always_inline)) {
        if constexpr (LISTED)
            if (wm == 0 && lane < C::BN && j < mine)
                copy4(a.list + k_first + min(tile_of(j) * C::BN + lane, reach.total - 1), (lds_char*)named[wk][j & 3]);
    };
    // row r of tile t, of round j, which need not be whole
    auto row_of = [&](int t, int j, int r) __attribute__((always_inline)) -> int64_t {
        // (sequences that overlap, against the call's contract, write over one another's lists, or leave some unwritten)
        if constexpr (LISTED) return min(max(named[wk][j & 3][r], 0), k_last);
        const int u = min(t * C::BN + r, reach.total - 1);
        if constexpr (CACHE) return slot_of(a, reach, u);
        return u;
    };
    // all copies of the keys or values of round j's tile
    auto copy = [&](int j, const char* from, auto value, lds_char* to) __attribute__((always_inline)) {
        constexpr bool V = decltype(value)::value;
        const uint32_t pitch = V ? pitch_v : pitch_k;
        const int t = tile_of(j);
        int row;
        if (whole(t, row)) {
            from += (int64_t)row * pitch;
#pragma unroll
            for (int i = 0; i < C::NC; ++i) {
                const int r = i * (WM * C::RPC) + row0;
                const uint32_t at = (pc ^ (V ? C::swap_v(r) : C::swap_k(r))) * 16;
                // (rows evenly apart: a scalar from copy to copy, and one offset for a lane)
                if constexpr (CACHE) copy16(from + (uint32_t)(r * pitch + at), to + (i * WM + wm) * 1024);
                else copy16(from + (int64_t)(i * (WM * C::RPC)) * pitch + (uint32_t)(row0 * pitch + at), to + (i * WM + wm) * 1024);
            }
        } else {
#pragma unroll (LISTED ? C::NC : 1)
            for (int i = 0; i < C::NC; ++i) {
                const int r = i * (WM * C::RPC) + row0;
                copy16(from + row_of(t, j, r) * pitch + (pc ^ (V ? C::swap_v(r) : C::swap_k(r))) * 16,
                       to + (i * WM + wm) * 1024);
            }
        }
    };
    // PL: a thread's pieces of round j's tile, and their planes into LDS
    auto fetch = [&](int j, const char* from, uint32_t pitch, uint4 (&g)[C::NG > 0 ? C::NG : 1])
        __attribute__((always_inline)) {
        const int t = tile_of(j);
        int row;
        if (whole(t, row)) {
            from += (int64_t)row * pitch;
#pragma unroll
            for (int i = 0; i < C::NG; ++i) {
                const uint32_t at = threadIdx.x + 256 * i;
                if constexpr (CACHE) g[i] = *(const uint4*)(from + at * 16);
                else g[i] = *(const uint4*)(from + at / (C::RB / 16) * pitch + at % (C::RB / 16) * 16);
            }
        } else {
#pragma unroll
            for (int i = 0; i < C::NG; ++i) {
                const int at = threadIdx.x + 256 * i, r = at / (C::RB / 16), p = at % (C::RB / 16);
                g[i] = *(const uint4*)(from + p * 16 + row_of(t, j, r) * pitch);
            }
        }
    };
    bool bad = false;
    auto spread = [&](const uint4 g, int i, auto value, lds_char* to) __attribute__((always_inline)) {
        constexpr bool V = decltype(value)::value;
        typedef uint32_t u2v __attribute__((ext_vector_type(2)));
        const int at = threadIdx.x + 256 * i, r = at / (C::RB / 16), p = at % (C::RB / 16);
        bad |= special(g);
        uint32_t w[3][2];
        cut_pair(g.x, g.y, w[0][0], w[1][0], w[2][0]);
        cut_pair(g.z, g.w, w[0][1], w[1][1], w[2][1]);
        lds_char* dst = to + r * C::LRB + ((p >> 1) ^ (V ? C::swap_v(r) : C::swap_k(r))) * 16 + (p & 1) * 8;
#pragma unroll
        for (int q = 0; q < 3; ++q) *(__attribute__((address_space(3))) u2v*)(dst + q * C::PB) = u2v{w[q][0], w[q][1]};
    };
    auto meet = [&]() __attribute__((always_inline)) {
        wait_vm<0>();
        // a wavefront with tiles of its own waits for no one
        if (WM > 1) lds_barrier();
        else asm volatile("" ::: "memory");
    };
    // zeros in the place of a tile of values, for a group that goes round without one
    auto no_values = [&](lds_char* to) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < C::NC; ++j) copy16(attend_zero, to + (j * WM + wm) * 1024);
    };
    lds_char* const kbuf = own;
    lds_char* const vbuf = own + 2 * C::TB;

    constexpr int STEPS = C::NT * C::QN;               // of the product with the keys
    struct Operand {
        uint4 p[C::NP];
    };
    auto key_step = [&](f16v (&s)[C::NT], int i, const Operand& k) __attribute__((always_inline)) {
        const int t = i / C::QN, c = i % C::QN;
        if constexpr (C::PL) {
            s[t] = mfma_planes(k.p, qf[c], s[t]);
        } else if constexpr (F32) {
            const uint4 kf = k.p[0], q = qf[c][0];
            const uint32_t kv[4] = {kf.x, kf.y, kf.z, kf.w}, qv[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                s[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kv[e]), __uint_as_float(qv[e]), s[t], 0, 0, 0);
        } else {
            s[t] = mfma32(k.p[0], qf[c][0], s[t]);
        }
    };
    auto key_load = [&](const lds_char* kl, int i) __attribute__((always_inline)) {
        const int r = 32 * (i / C::QN) + col;
        Operand k;
#pragma unroll
        for (int p = 0; p < C::NP; ++p)
            k.p[p] = lds16(kl + p * C::PB + r * C::LRB + ((2 * (i % C::QN) + h) ^ C::swap_k(r)) * 16);
        return k;
    };
    auto clear = [&](f16v (&s)[C::NT]) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < C::NT; ++t) s[t] = f16v{};
    };

    // Round j: the softmax of tile j's scores s beside the products that give tile
    // j + 1's, in n (a wavefront's vector instructions run while its matrix
    // instructions do, if they are next to each other), then the product with the
    // values.  P: j & 1.
    auto round = [&](int j, auto parity, f16v (&s)[C::NT], f16v (&n)[C::NT]) __attribute__((always_inline)) {
        constexpr int P = decltype(parity)::value;
        meet();
        uint4 gk[C::NG > 0 ? C::NG : 1], gv[C::NG > 0 ? C::NG : 1];
        if (j + 2 < mine) {
            if constexpr (C::PL) fetch(j + 2, kg, pitch_k, gk);
            else copy(j + 2, kg, std::false_type{}, kbuf + P * C::TB);
        }
        name(j + 3);
        if (j + 1 < mine) {
            if constexpr (C::PL) fetch(j + 1, vg, pitch_v, gv);
            else copy(j + 1, vg, std::true_type{}, vbuf + (1 - P) * C::TB);
        } else if (WM == 2 && j + 1 < rounds) {
            no_values(vbuf + (1 - P) * C::TB);
        }
        const lds_char* kl = kbuf + (1 - P) * C::TB;
        const lds_char* vl = vbuf + P * C::TB;
        const int u0 = tile_of(j) * C::BN;
        clear(n);
        // A tile that the wavefront does not see at all goes the same way (skipping it cost registers, and it spilled), and
        // so does the round in which a group has none: whatever its scores are they are left out, and its values are zeros
        // (what the buffer held before must not be looked at: it would decide on `again`).
        const bool masked = j >= mine || u0 + C::BN - 1 > wl_first || (u0 < wf_last && u0 + C::BN > a.sinks);
        if (masked) {
#pragma unroll
            for (int t = 0; t < C::NT; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int u = u0 + 32 * t + 8 * (e >> 2) + 4 * h + (e & 3);
                    s[t][e] = j < mine && u <= last && (u >= from || u < a.sinks) ? s[t][e] : -INFINITY;
                }
        }
        if (!C::PL && masked) {
            // A masked key's probability is zero, but its values may be infinite
            // or NaN, and the matrix product would carry those to every row.
            // (Planes find them as they are split, in every tile.)
            uint32_t big = 0;
#pragma unroll 2
            for (int i = lane; i < C::TB / 16; i += 64) {
                const uint4 v = lds16(vl + i * 16);
                for (uint32_t w : {v.x, v.y, v.z, v.w}) {
                    if constexpr (F32) big |= (w & 0x7F800000u) == 0x7F800000u;
                    else big |= ((w & 0x7F80u) == 0x7F80u) | ((w & 0x7F800000u) == 0x7F800000u);
                }
            }
            again |= __ballot(big != 0) != 0;
        }
        // (past the last tile these are products of what the buffer holds; nobody reads them)
        constexpr int FIRST = STEPS / 4;
        // operands under way: LDS answers after about four products
        constexpr int KA = C::PL || STEPS < 4 ? 2 : 4;
        Operand kf[KA];
#pragma unroll
        for (int i = 0; i < KA - 1; ++i) kf[i] = key_load(kl, i);
        auto key_next = [&](int i) __attribute__((always_inline)) {
            if (i + KA - 1 < STEPS) kf[(i + KA - 1) % KA] = key_load(kl, i + KA - 1);
            key_step(n, i, kf[i % KA]);
        };
#pragma unroll
        for (int i = 0; i < FIRST; ++i) key_next(i);
        float mx = s[0][0];
#pragma unroll
        for (int t = 0; t < C::NT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[t][e]);
        {
            const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            mx = fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1])) * a.scale;
        }
        // m is the reference of the row's exponents: a probability may be up to 2^8
        // before it moves, so that the sums are hardly ever scaled again.  Rows that
        // need not move keep theirs (scaled by 1): their bits are not the others' concern.
        if (__ballot(mx > m + 8.f) != 0) {
            asm volatile("");                          // a branch: the compiler would scale by 1 instead
            const float mn = mx > m + 8.f ? mx : m;
            const float alpha = __builtin_amdgcn_exp2f(m - (mn == -INFINITY ? 0.f : mn));
            m = mn;
            l *= alpha;
#pragma unroll
            for (int t = 0; t < D / 32; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[t][e] *= alpha;
        }
        const float ms = m == -INFINITY ? 0.f : m;
        uint4 pf[C::NT * 2][PP];                       // bf16 operands: eight probabilities each
        // the values of 16 keys (bf16 operands) or of two (fp32), all of a head
        constexpr int VS = C::B16 ? C::BN / 16 : 16, VA = C::B16 ? 2 : 4;
        Operand vf[VA][D / 32];
        auto value_load = [&](int ks) __attribute__((always_inline)) {
            if constexpr (!C::B16) {
                const int key = 8 * (ks >> 2) + 4 * h + (ks & 3);
#pragma unroll
                for (int t = 0; t < D / 32; ++t) {
                    const int at = key * C::RB + (((8 * t + col / 4) ^ C::swap_v(key)) * 4 + col % 4) * 4;
                    vf[ks % VA][t].p[0].x = *(const __attribute__((address_space(3))) uint32_t*)(vl + at);
                }
            } else {
                const int i = lane & 15, key = 16 * ks + 4 * h + (i >> 2);
                // rows key and key + 8 have the same swap
                const lds_char* at = vl + key * C::LRB + 8 * (i & 1);
#pragma unroll
                for (int t = 0; t < D / 32; ++t)
#pragma unroll
                    for (int p = 0; p < C::NP; ++p) {
                        const int c = (4 * t + 2 * ((lane >> 4) & 1) + ((i >> 1) & 1)) ^ C::swap_v(key);
                        typedef __attribute__((address_space(3))) s4v lds_s4v;
                        const s4v v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v*)(at + p * C::PB + c * 16));
                        const s4v v1 =
                            __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v*)(at + p * C::PB + 8 * C::LRB + c * 16));
                        __builtin_memcpy(&vf[ks % VA][t].p[p], &v0, 8);
                        __builtin_memcpy((char*)&vf[ks % VA][t].p[p] + 8, &v1, 8);
                    }
            }
        };
        constexpr int ALL = 16 * C::NT, LEFT = STEPS - FIRST;
#pragma unroll
        for (int i = 0; i < LEFT; ++i) {
            if (i == LEFT - (LEFT + 3) / 4) value_load(0);
            key_next(FIRST + i);
#pragma unroll
            for (int e = i * ALL / LEFT; e < (i + 1) * ALL / LEFT; ++e) {
                const float x = __builtin_amdgcn_exp2f(fmaf(s[e >> 4][e & 15], a.scale, -ms));
                s[e >> 4][e & 15] = x;
                l += x;
                if (C::B16 && (e & 1)) {
                    uint32_t w[3];
                    if constexpr (C::PL)
                        cut_pair(__float_as_uint(s[e >> 4][(e & 15) - 1]), __float_as_uint(x), w[0], w[1], w[2]);
                    else if constexpr (PP == 2)
                        two_parts(s[e >> 4][(e & 15) - 1], x, w[0], w[1]);
                    else
                        w[0] = bf16_pair(s[e >> 4][(e & 15) - 1], x);
#pragma unroll
                    for (int p = 0; p < PP; ++p) {
                        uint4& f = pf[e >> 3][p];
                        if ((e & 7) == 1) f.x = w[p];
                        else if ((e & 7) == 3) f.y = w[p];
                        else if ((e & 7) == 5) f.z = w[p];
                        else f.w = w[p];
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int d = 1; d < VA - 1; ++d) value_load(d);
#pragma unroll
        for (int ks = 0; ks < VS; ++ks) {
            if (ks + VA - 1 < VS) value_load(ks + VA - 1);
#pragma unroll
            for (int t = 0; t < D / 32; ++t) {
                const Operand& v = vf[ks % VA][t];
                if constexpr (PP == 2) o[t] = mfma32(v.p[0], pf[ks][1], o[t]);
                if constexpr (C::PL) o[t] = mfma_planes(v.p, pf[ks], o[t]);
                else if constexpr (F32)
                    o[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(v.p[0].x), s[0][ks], o[t], 0, 0, 0);
                else o[t] = mfma32(v.p[0], pf[ks][0], o[t]);
            }
            if constexpr (C::PL) {
                // the next tiles' planes beside the products
#pragma unroll
                for (int i = ks * C::NG / VS; i < (ks + 1) * C::NG / VS; ++i) {
                    if (j + 2 < mine) spread(gk[i], i, std::false_type{}, kbuf + P * C::TB);
                    if (j + 1 < mine) spread(gv[i], i, std::true_type{}, vbuf + (1 - P) * C::TB);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    f16v sa[C::NT], sb[C::NT];
    clear(sa);
    auto first_copy = [&](int j, const char* from, auto value, lds_char* to) __attribute__((always_inline)) {
        if constexpr (C::PL) {
            uint4 g[C::NG];
            fetch(j, from, decltype(value)::value ? pitch_v : pitch_k, g);
#pragma unroll
            for (int i = 0; i < C::NG; ++i) spread(g[i], i, value, to);
        } else {
            copy(j, from, value, to);
        }
    };
    if constexpr (LISTED) {
        for (int j = 0; j < 3; ++j) name(j);
        meet();
    }
    if (mine > 0) first_copy(0, kg, std::false_type{}, kbuf);
    meet();
    if (WM == 2 && mine == 0 && rounds > 0) no_values(vbuf);
    if (mine > 0) {
        first_copy(0, vg, std::true_type{}, vbuf);
        if (mine > 1) first_copy(1, kg, std::false_type{}, kbuf + C::TB);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) key_step(sa, i, key_load(kbuf, i));
    }
    for (int j = 0; j < rounds; j += 2) {
        round(j, std::integral_constant<int, 0>{}, sa, sb);
        if (j + 1 < rounds) round(j + 1, std::integral_constant<int, 1>{}, sb, sa);
    }
    if constexpr (C::PL) {
        // a wavefront's share of the keys and values is every wavefront's concern
        const float any = __ballot(bad) != 0 ? 1.f : 0.f;
        if (lane == 0) ml[wave][0][0] = any;
        __syncthreads();
#pragma unroll
        for (int g = 0; g < 4; ++g) again |= ml[g][0][0] != 0.f;
    }
    if (again) {
        // Keys one by one, each only for the rows that see it: the wavefront's
        // sums formed again from the cache.
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int t = 0; t < D / 32; ++t) o[t] = f16v{};
        const char* qr = query;
#pragma unroll 1
        for (int u = tb * C::BN; u < min(te * C::BN, reach.total); ++u) {
            if ((u / C::BN - tb) % C::WK != wk || !(u <= last && (u >= from || u < a.sinks))) continue;
            int64_t at = u;
            if constexpr (CACHE) at = slot_of(a, reach, u);
            if constexpr (LISTED) at = min(max(a.list[k_first + u], 0), k_last);
            float x = 0.f;
#pragma unroll 1
            for (int c = 0; c < C::RB / 16; ++c) {
                uint4 qv = *(const uint4*)(qr + c * 16), kv = *(const uint4*)(kg + at * pitch_k + c * 16);
                const uint32_t qw[4] = {qv.x ^ a.flip, qv.y ^ a.flip, qv.z ^ a.flip, qv.w ^ a.flip};
                const uint32_t kw[4] = {kv.x, kv.y, kv.z, kv.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (F32) {
                        x = fmaf(__uint_as_float(qw[e]), __uint_as_float(kw[e]), x);
                    } else {
                        x = fmaf(__uint_as_float(qw[e] << 16), __uint_as_float(kw[e] << 16), x);
                        x = fmaf(__uint_as_float(qw[e] & 0xFFFF0000u), __uint_as_float(kw[e] & 0xFFFF0000u), x);
                    }
                }
            }
            x *= a.scale;
            const float mn = fmaxf(m, x), ms = mn == -INFINITY ? 0.f : mn;
            const float alpha = __builtin_amdgcn_exp2f(m - ms), p = __builtin_amdgcn_exp2f(x - ms);
            m = mn;
            l = fmaf(l, alpha, p);
            const char* vr = vg + at * pitch_v;
#pragma unroll
            for (int e = 0; e < C::ON; ++e) {
                const int d = 32 * (e >> 4) + 8 * ((e >> 2) & 3) + 4 * h + (e & 3);
                const float v = F32 ? ((const float*)vr)[d] : __uint_as_float((uint32_t)((const uint16_t*)vr)[d] << 16);
                o[e >> 4][e & 15] = fmaf(p, v, o[e >> 4][e & 15] * alpha);
            }
        }
        if (h == 1) l = 0.f;                           // both lanes of a row have all of its sum
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
        __syncthreads();               // all tiles have been read, too
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
    // a row that sees no key has zeros: its sum is told from one of scores of minus infinity by its sign
    if (!CACHE && reach.total == 0) l = -0.f;
    const float r = a.splits > 1 ? 1.f : !CACHE && reach.total == 0 ? 0.f : 1.f / l;
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

constexpr int MAX_SPLITS = 64;

// The splits' sums of one row, joined by a wavefront: lane s forms split s's
// weight, then groups of D / 4 lanes take every (256 / D)th split's sums, four of
// them under way, and are added up.  (Splits one after the other in one group of
// lanes: 9.3 us for 17 of them, against 7.7 for the attention itself.)
template <bool F32, int D, bool CACHE>
__global__ __launch_bounds__(256) void join_kernel(const float* part, void* out, int64_t rows, int splits, int heads,
                                                   const int32_t* end) {
    constexpr int G = 256 / D;                         // groups
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows || (end && row >= (int64_t)*end * heads)) return;
    const int lane = threadIdx.x & 63, d = lane % (D / 4) * 4, g = lane / (D / 4);
    const float* from = part + row * D + d;
    float2 ml = make_float2(-INFINITY, CACHE ? 0.f : -0.f);
    if (lane < splits) ml = *(const float2*)(part + splits * rows * D + (lane * rows + row) * 2);
    float big = ml.x;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) big = fmaxf(big, __shfl_xor(big, i));
    const float f = __builtin_amdgcn_exp2f(ml.x - (big == -INFINITY ? 0.f : big));
    float l = f * ml.y;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) l += __shfl_xor(l, i);
    f4v v = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < splits; s0 += 4 * G) {
        f4v p[4];
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = s0 + i * G + g;
            p[i] = s < splits ? *(const f4v*)(from + s * rows * D) : f4v{0.f, 0.f, 0.f, 0.f};
            w[i] = __shfl(f, min(s, MAX_SPLITS - 1));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fmaf(w[i], p[i][e], v[e]);
    }
    // (sums of minus zero alone: the row sees no key)
    const float r = !CACHE && __float_as_uint(l) == 0x80000000u ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int i = D / 4; i < 64; i <<= 1) v[e] += __shfl_xor(v[e], i);
        v[e] *= r;
    }
    if (g != 0) return;
    if constexpr (F32) *(f4v*)((float*)out + row * D + d) = v;
    else *(uint2*)((uint16_t*)out + row * D + d) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
}

// Where the device says how many rows of a call its sequences have.
inline const int32_t* rows_end(const TokenRows& r) { return r.start ? r.start + r.batch : nullptr; }

// Workgroups of attend_kernel that a compute unit is asked to take (the launch bounds).  Registers and LDS leave room
// for more in places: two of fp32 heads of 64 with WM 2 and 4, three or four of heads of 32.
template <bool F32, int D>
int attend_places(int wm) {
    if constexpr (!(F32 && D == 128))
        if (wm == 1) return AttendShape<F32, D, 1>::WGS;
    return wm == 2 ? AttendShape<F32, D, 2>::WGS : AttendShape<F32, D, 4>::WGS;
}

inline int attend_places(bool f32, int dim, int wm) {
    if (f32) return dim == 32 ? attend_places<true, 32>(wm) : dim == 64 ? attend_places<true, 64>(wm) : attend_places<true, 128>(wm);
    return dim == 32 ? attend_places<false, 32>(wm) : dim == 64 ? attend_places<false, 64>(wm) : attend_places<false, 128>(wm);
}

// How a call is cut up, from what the host knows.
struct AttendCut {
    int wm, qtiles, splits;
    int64_t grid;
};

// rows: of a sequence and key head, at most; heads: key heads of all sequences; keys: of a sequence, at most; uneven:
// sequences may be much shorter than that
inline void cut_keys(AttendCut* cut, bool f32, int dim, int64_t rows, int64_t heads, int64_t keys, bool uneven) {
    // fp32 heads of 128 values: two tiles of keys and of values for each of four wavefronts would not fit
    cut->wm = rows <= 32 && !(f32 && dim == 128) ? 1 : rows <= 64 ? 2 : 4;
    cut->qtiles = (int)((rows + 32 * cut->wm - 1) / (32 * cut->wm));
    const int64_t base = (int64_t)cut->qtiles * heads;
    const int bn = (cut->wm == 1 || (f32 && !(cut->wm == 4 && dim == 32)) ? 32 : 64) * (4 / cut->wm);
    // Splits of the keys, of two tiles for each group at least.  Few rows are bound by the cache's bytes: two workgroups
    // for every compute unit.  Otherwise the number that makes the share of a full card times its passes least; each
    // split costs its sums' way through memory, about a hundredth (216 tiles of fp32: in three, 648 workgroups on 512
    // places, 942 us; in seven, three nearly full passes, 806).
    const int64_t most = std::max((int64_t)1, std::min((keys + 2 * bn - 1) / (2 * bn), (int64_t)MAX_SPLITS));
    cut->splits = 1;
    if (base > 0 && cut->wm == 1) {
        if (base < 256) cut->splits = (int)std::min((512 + base - 1) / base, most);
    } else if (base > 0) {
        const int64_t places = 256 * attend_places(f32, dim, cut->wm);
        double best = 0.;
        for (int64_t n = 1; base < 2 * places && n <= most; ++n) {
            const double cost = (double)((base * n + places - 1) / places) / n + (n > 1 ? 0.01 * n * base / places : 0.);
            if (n == 1 || cost < best) {
                best = cost;
                cut->splits = (int)n;
            }
        }
        // Of sequences whose lengths only the device knows the longest would be the time: three times as many workgroups as
        // places, so that the short ones' make room (nine of up to 257 queries and 12001 keys, four fp32 heads of 128 on
        // one, 166 us for 268).
        if (uneven) cut->splits = (int)std::max((int64_t)cut->splits, std::min((3 * places + base - 1) / base, most));
    }
    cut->grid = base * cut->splits;
}

}  // namespace ssc
