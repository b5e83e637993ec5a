// Attention of one set of tokens to another: a call's mask turned into lists of
// visible keys, and the attention kernel (attend_kernel.h) over the keys as they lie
// or over the listed ones.
//
// Keys have no order, so the visible ones of a sequence may as well be the only
// ones: their rows' numbers, one behind the other, are all that the attention looks
// at, and cells that are not visible cost nothing but the reading of their byte of the
// mask.
//
// Bound by the softmax's vector instructions and the products with the values, twice as
// many as with the keys (3600 queries, a quarter of four times 53568 cells visible, 8
// bf16 heads of 32: 161 us; all cells, 16 heads of 64 on 4: 1370 us, 577 TFLOP/s of the
// formula's; with probabilities rounded to bf16 117 and 980).  Matrix cores are busy 21
// and 37 % of the time.
#include "attend_kernel.h"

#include <algorithm>
#include <cmath>
#include <limits>

namespace ssc {

constexpr int LIST_KEYS = 4096;                        // of a workgroup: four each of 1024 threads

// Which bytes of a word are not zero, a bit each.
__device__ __forceinline__ uint32_t seen4(uint32_t w) {
    const uint32_t x = (((w & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | w) & 0x80808080u;
    return x * 0x00204081u >> 28;
}

// The sequence and the part of it that workgroup `slot` has, where sequence b's parts are first / LIST_KEYS + b onwards, as
// many as it needs at most; false: none.
__device__ __forceinline__ int list_slot(int first, int b) { return first / LIST_KEYS + b; }

__device__ __forceinline__ bool list_part(const TokenRows& keys, int slot, int& b, int& part, int& first, int& n) {
    int lo = 0, hi = keys.batch - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        rows_of(keys, mid, first, n);
        if (list_slot(first, mid) <= slot) lo = mid; else hi = mid - 1;
    }
    b = lo;
    rows_of(keys, b, first, n);
    const int p = slot - list_slot(first, b);
    if (p < 0 || p >= (n + LIST_KEYS - 1) / LIST_KEYS) return false;
    part = p * LIST_KEYS;
    return true;
}

// How many keys of a part are visible.
__global__ __launch_bounds__(256) void count_kernel(const uint8_t* mask, TokenRows keys, int32_t* counts, int64_t id0) {
    __shared__ int sums[4];
    const int slot = (int)(id0 + blockIdx.x), t = threadIdx.x;
    int b, part, first, n;
    if (!list_part(keys, slot, b, part, first, n)) return;
    mask += first;
    const int at = part + 16 * t;
    int seen = 0;
    if (at + 16 <= n) {
        uint32_t w[4];
        __builtin_memcpy(w, mask + at, 16);
        seen = __popc(seen4(w[0])) + __popc(seen4(w[1])) + __popc(seen4(w[2])) + __popc(seen4(w[3]));
    } else {
        for (int i = at; i < n; ++i) seen += mask[i] != 0;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) seen += __shfl_xor(seen, o);
    if ((t & 63) == 0) sums[t >> 6] = seen;
    __syncthreads();
    if (t == 0) counts[slot] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// The counts of a sequence's parts made those of the parts before, a wavefront a sequence, four parts a lane; and the
// sequence's own.
__global__ __launch_bounds__(256) void before_kernel(TokenRows keys, int32_t* counts, int32_t* count) {
    const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (id >= keys.batch) return;
    int first, n;
    rows_of(keys, (int)id, first, n);
    const int parts = (n + LIST_KEYS - 1) / LIST_KEYS;
    counts += list_slot(first, (int)id);
    uint32_t all = 0;
    for (int i = 4 * lane; i - 4 * lane < parts; i += 256) {
        uint32_t c[4], mine = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            c[e] = i + e < parts ? (uint32_t)counts[i + e] : 0;
            mine += c[e];
        }
        uint32_t upto = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t v = __shfl_up(upto, o);
            if (lane >= o) upto += v;
        }
        uint32_t before = all + upto - mine;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (i + e < parts) counts[i + e] = (int)before;
            before += c[e];
        }
        all += __shfl(upto, 63);
    }
    if (lane == 0) count[id] = (int)min(all, (uint32_t)n);
}

// A sequence's visible keys in order.  Workgroup b * parts + p lists those among the p-th
// LIST_KEYS of sequence b, behind the ones before them.  Of few parts it counts those
// itself, 16 bytes a lane: further launches would take longer than reading a mask again
// (four maps of 53568 cells 5 us).  COUNTED: of many the two kernels above have, and
// workgroup `slot` has what list_part() says.
template <bool COUNTED>
__global__ __launch_bounds__(1024) void list_kernel(const uint8_t* mask, TokenRows keys, int32_t* list, int32_t* count,
                                                    const int32_t* counts, int parts, int64_t id0) {
    __shared__ int sums[2][16];
    const int64_t id = id0 + blockIdx.x;
    const int t = threadIdx.x;
    int b, part, first, n;
    if constexpr (COUNTED) {
        if (!list_part(keys, (int)id, b, part, first, n)) return;
    } else {
        b = (int)(id / parts);
        part = (int)(id % parts) * LIST_KEYS;
        rows_of(keys, b, first, n);
        if (part >= n && part > 0) return;
    }
    mask += first;
    const int at = part + 4 * t;
    uint32_t word = 0;
    if (at + 4 <= n) {
        __builtin_memcpy(&word, mask + at, 4);
    } else {
        for (int i = 0; at + i < n; ++i) word |= (uint32_t)mask[at + i] << (8 * i);
    }
    int before = 0;
    if constexpr (!COUNTED) {
#pragma unroll 4
        for (int i = t * 16; i < part; i += 16 * 1024) {
            uint32_t w[4];
            __builtin_memcpy(w, mask + i, 16);
            before += __popc(seen4(w[0])) + __popc(seen4(w[1])) + __popc(seen4(w[2])) + __popc(seen4(w[3]));
        }
    }
    const uint32_t bits = seen4(word);
    const int mine = __popc(bits);
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        if constexpr (!COUNTED) before += __shfl_xor(before, o);
        const int v = __shfl_up(upto, o);
        if ((t & 63) >= o) upto += v;
    }
    if ((t & 63) == 63) {
        sums[0][t >> 6] = before;
        sums[1][t >> 6] = upto;
    }
    __syncthreads();
    int base = 0, all = 0;
    // (sequences that overlap, against the call's contract, count over one another's parts)
    if constexpr (COUNTED) base = min(max(counts[id], 0), part);
#pragma unroll
    for (int w = 0; w < 16; ++w) {
        base += sums[0][w] + (w < (t >> 6) ? sums[1][w] : 0);
        all += sums[0][w] + sums[1][w];
    }
    int32_t* to = list + first + base + upto - mine;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (bits >> i & 1) *to++ = at + i;
    if (!COUNTED && t == 0 && part + LIST_KEYS >= n) count[b] = all;
}

namespace {

// Parts of a sequence up to which each workgroup of a list counts for itself (one query over a sequence of 64 parts,
// counting itself 12.9 us, from counts 13.0; 128 parts 16.6 and 13.8; four sequences of 64 parts 13.6 and 15.1, of 128
// 24.7 and 16.5; the counting grows with the square of the keys: 2^28 of them 1144 ms, from
// counts 0.6).
constexpr int COUNT_PARTS = 64;
// Where the longest sequence is not known, or much longer than the others, most workgroups have no part; so many, and for
// each that may have one so many more, are left to find that out (100 sequences with 209000 keys in all, 5100 workgroups
// for 150: counting itself 22.3 us, from counts 26.8; 300, 15900 for 350: 35.4 and 23.8; 20000, 940000 for 20046: 1552 and
// 317; 100000 with 150000 keys 6190 and 1640).
constexpr int64_t COUNT_SPARE = 8192, COUNT_SPARE_EACH = 8;

// What a call needs of its workspace: the splits' sums, the lists, their lengths, their parts' counts.
struct CrossPlan {
    AttendCut cut;
    int queries, keys;     // rows that the sequences can have
    int64_t slots;         // of parts, where they are counted first
    size_t list, all;
};

bool cross_plan(const sscater_cross_spec* s, bool masked, CrossPlan* p) {
    if (!s || (s->dtype != SSCATER_F32 && s->dtype != SSCATER_BF16)) return false;
    if (s->batch < 1 || s->batch > (1 << 24) || s->kv_heads < 1 || s->q_heads < 1 || s->q_heads > (1 << 16) ||
        s->q_heads % s->kv_heads || (s->head_dim != 32 && s->head_dim != 64 && s->head_dim != 128))
        return false;
    if (!(s->scale == s->scale) || s->rounded < 0 || s->rounded > 1 || (s->q_start == nullptr) != (s->k_start == nullptr) || (uintptr_t)s->q_start % 4 ||
        (uintptr_t)s->k_start % 4)
        return false;
    auto rows_ok = [&](int64_t all, int64_t most) {
        return all >= 0 && all <= (1 << 30) && most >= 0 && most <= all && (s->q_start || most * s->batch == all);
    };
    if (!rows_ok(s->queries, s->max_q) || !rows_ok(s->keys, s->max_k)) return false;
    const int64_t size = s->dtype == SSCATER_F32 ? 4 : 2, q = (int64_t)s->q_heads * s->head_dim,
                  kv = (int64_t)s->kv_heads * s->head_dim, most = 1 << 24;
    if (s->q_stride < q || s->k_stride < kv || s->v_stride < kv || s->q_stride > most || s->k_stride > most ||
        s->v_stride > most || s->q_stride * size % 16 || s->k_stride * size % 16 || s->v_stride * size % 16)
        return false;
    const int64_t rows = (int64_t)s->max_q * (s->q_heads / s->kv_heads);
    if (rows > (1 << 30) || (int64_t)s->queries * s->q_heads > (int64_t(1) << 40)) return false;
    cut_keys(&p->cut, s->dtype == SSCATER_F32, s->head_dim, rows, (int64_t)s->kv_heads * s->batch, s->max_k,
             s->batch > 1 && s->q_start != nullptr);
    if (p->cut.grid > 0x7FFFFFFF) return false;
    p->queries = (int)std::min((int64_t)s->queries, (int64_t)s->max_q * s->batch);
    p->keys = (int)std::min((int64_t)s->keys, (int64_t)s->max_k * s->batch);
    p->list = p->cut.splits > 1 ? (size_t)p->cut.splits * p->queries * s->q_heads * (s->head_dim + 2) * 4 : 0;
    p->list = (p->list + 15) / 16 * 16;
    p->slots = (int64_t)p->keys / LIST_KEYS + s->batch;
    const int64_t parts = ((int64_t)s->max_k + LIST_KEYS - 1) / LIST_KEYS;
    if (parts <= COUNT_PARTS && parts * s->batch <= COUNT_SPARE + COUNT_SPARE_EACH * p->slots) p->slots = 0;
    p->all = p->list + (masked && p->keys > 0 ? ((size_t)p->keys + s->batch + p->slots) * 4 : 0);
    return true;
}

template <bool F32, int D, Keys SRC, bool ONE>
void launch_cross(AttendArgs a, const AttendCut& cut, hipStream_t s) {
    const dim3 block(256);
    for (int64_t at = 0; at < cut.grid; at += LAUNCH_GROUPS) {
        a.id0 = (int)at;
        const dim3 grid((unsigned)std::min(LAUNCH_GROUPS, cut.grid - at));
        if constexpr (!(F32 && D == 128) && !ONE) {
            if (cut.wm == 1) attend_kernel<F32, D, 1, SRC, false><<<grid, block, 0, s>>>(a);
        }
        if (cut.wm == 2) attend_kernel<F32, D, 2, SRC, ONE><<<grid, block, 0, s>>>(a);
        if (cut.wm == 4) attend_kernel<F32, D, 4, SRC, ONE><<<grid, block, 0, s>>>(a);
    }
    if (cut.splits > 1) {                              // at most some hundred thousand rows: see cut_keys
        const int64_t rows = (int64_t)a.rows.tokens * a.q_heads;
        join_kernel<F32, D, false><<<dim3((unsigned)((rows + 3) / 4)), block, 0, s>>>(a.part, a.out, rows, cut.splits,
                                                                                      a.q_heads, rows_end(a.rows));
    }
}

template <bool F32, Keys SRC, bool ONE>
void launch_cross(const AttendArgs& a, const AttendCut& cut, int dim, hipStream_t s) {
    if (dim == 32) launch_cross<F32, 32, SRC, ONE>(a, cut, s);
    else if (dim == 64) launch_cross<F32, 64, SRC, ONE>(a, cut, s);
    else launch_cross<F32, 128, SRC, ONE>(a, cut, s);
}

template <Keys SRC>
void launch_cross(const AttendArgs& a, const AttendCut& cut, bool f32, bool one, int dim, hipStream_t s) {
    if (f32) launch_cross<true, SRC, false>(a, cut, dim, s);
    else if (one && cut.wm > 1) launch_cross<false, SRC, true>(a, cut, dim, s);
    else launch_cross<false, SRC, false>(a, cut, dim, s);
}

}  // namespace

}  // namespace ssc

using namespace ssc;

extern "C" {

int sscater_cross_workspace(const sscater_cross_spec* spec, int32_t masked, size_t* bytes) {
    CrossPlan p;
    if (!bytes || masked < 0 || masked > 1 || !cross_plan(spec, masked != 0, &p)) return SSCATER_E_INVALID_ARG;
    *bytes = p.all;
    return SSCATER_OK;
}

int sscater_cross_attend(const sscater_cross_spec* spec, const void* q, const void* k, const void* v,
                         const uint8_t* mask, void* out, void* workspace, size_t workspace_bytes, void* stream) {
    CrossPlan p;
    if (!cross_plan(spec, mask != nullptr, &p)) return SSCATER_E_INVALID_ARG;
    if (p.queries == 0) return SSCATER_OK;
    for (const void* x : {q, (const void*)out})
        if (!x || (uintptr_t)x % 16) return SSCATER_E_INVALID_ARG;
    for (const void* x : {k, v})
        if ((!x && p.keys > 0) || (uintptr_t)x % 16) return SSCATER_E_INVALID_ARG;
    if (p.all > 0 && (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < p.all)) return SSCATER_E_INVALID_ARG;
    const bool f32 = spec->dtype == SSCATER_F32, listed = mask != nullptr && p.keys > 0;
    const uint32_t size = f32 ? 4 : 2;
    AttendArgs a{};
    a.rows.tokens = p.queries; a.rows.max_new = spec->max_q; a.rows.batch = spec->batch;
    a.rows.start = spec->q_start; a.rows.past = nullptr;
    a.q = q; a.k = k; a.v = v; a.out = out; a.part = (float*)workspace;
    a.q_heads = spec->q_heads; a.kv_heads = spec->kv_heads; a.group = spec->q_heads / spec->kv_heads;
    a.qtiles = p.cut.qtiles; a.splits = p.cut.splits;
    // not zero, so that a masked score times it stays -inf; the least number of all, times a finite score, is zero beside 1
    a.scale = std::max(std::fabs(spec->scale) * 1.4426950408889634f, std::numeric_limits<float>::denorm_min());
    a.flip = spec->scale < 0.f ? f32 ? 0x80000000u : 0x80008000u : 0u;
    a.pitch_q = spec->q_stride * size;
    a.pitch_k = (uint32_t)spec->k_stride * size; a.pitch_v = (uint32_t)spec->v_stride * size;
    a.keys = p.keys; a.max_k = spec->max_k; a.k_start = spec->k_start;
    if (listed) {
        int32_t* list = (int32_t*)((char*)workspace + p.list);
        a.list = list;
        a.count = list + p.keys;
        TokenRows keys;
        keys.tokens = p.keys; keys.max_new = spec->max_k; keys.batch = spec->batch; keys.start = spec->k_start;
        keys.past = nullptr;
        const hipStream_t on = (hipStream_t)stream;
        int32_t *const count = list + p.keys, *const counts = count + spec->batch;
        if (p.slots) {
            for (int64_t id = 0; id < p.slots; id += LAUNCH_GROUPS)
                count_kernel<<<dim3((unsigned)std::min(LAUNCH_GROUPS, p.slots - id)), dim3(256), 0, on>>>(mask, keys, counts, id);
            before_kernel<<<dim3((unsigned)((spec->batch + 3) / 4)), dim3(256), 0, on>>>(keys, counts, count);
        }
        const int64_t parts = std::max(1, (spec->max_k + LIST_KEYS - 1) / LIST_KEYS), groups = p.slots ? p.slots : parts * spec->batch;
        constexpr int64_t LAUNCH = LAUNCH_GROUPS / 4;  // workgroups of 1024 threads
        for (int64_t id = 0; id < groups; id += LAUNCH) {
            const dim3 grid((unsigned)std::min(LAUNCH, groups - id)), block(1024);
            if (p.slots) list_kernel<true><<<grid, block, 0, on>>>(mask, keys, list, count, counts, 0, id);
            else list_kernel<false><<<grid, block, 0, on>>>(mask, keys, list, count, nullptr, (int)parts, id);
        }
    }
    const bool one = spec->rounded != 0;
    if (listed) launch_cross<Keys::LISTED>(a, p.cut, f32, one, spec->head_dim, (hipStream_t)stream);
    else launch_cross<Keys::ROWS>(a, p.cut, f32, one, spec->head_dim, (hipStream_t)stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSCATER_OK : report_hip_error(e);
}

}  // extern "C"
