// What the token operators share: the cache's slots and the rows of a call.
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/sscater.h"
#include "device_common.h"

namespace ssc {

struct TokenRows {
    int tokens, max_new, batch;
    const int32_t* start;
    const int64_t* past;
};

// First row and number of new tokens of sequence b, inside the call's rows
// whatever start holds.
__device__ __forceinline__ void rows_of(const TokenRows& r, int b, int& first, int& n) {
    if (r.start) {
        first = min(max(r.start[b], 0), r.tokens);
        n = min(min(max(r.start[b + 1], first), r.tokens) - first, r.max_new);
    } else {
        first = b * r.max_new;
        n = r.max_new;
    }
}

__device__ __forceinline__ int64_t past_of(const TokenRows& r, int b) {
    const int64_t p = r.past[b];
    return p > 0 ? p : 0;
}

// Checks of the parts that several calls take; nullptr-safe.
bool token_cache_ok(const sscater_token_cache* c);
bool token_rows_ok(const sscater_token_cache* c, const sscater_token_rows* r);
TokenRows token_rows(const sscater_token_cache* c, const sscater_token_rows* r);

}  // namespace ssc
