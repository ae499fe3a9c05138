// Packed new tokens of several requests: what the calls on them share.
#pragma once
#include "common.cuh"

namespace sdv {

constexpr int kMaxRequests = 8192;             // requests of a call: their prefix sums stand in shared memory
constexpr int kMaxPoolBlocks = 1 << 25;        // so that a slot (64 x block + offset) is an int32

// Request b's new tokens (packed rows start .. end) behind its cached ones, and whether its blocks hold them all.
struct RequestSpan { int len, n; bool covered; };
__device__ __forceinline__ RequestSpan request_span(const sd_prompts& p, int b, int start, int end) {
    RequestSpan r;
    r.len = __ldcg(p.len + b);
    r.n = end - start;
    const long long blocks = ((long long)r.len + r.n + kBlock - 1) / kBlock;
    const int held = p.n_blocks ? min(__ldcg(p.n_blocks + b), p.max_blocks_per_seq) : p.max_blocks_per_seq;
    r.covered = r.len >= 0 && r.n == __ldcg(p.n_new + b) && blocks <= held;
    return r;
}

}  // namespace sdv
